"""Cases for the operators around a vocabulary-parallel head: the embedding lookup in its shards and the gradient for them, layer norm in front of
it (forward and backward), and the verification of drafted tokens on its logits.

Each case is one call as a serving loop or a training step makes it: `op` says which operator, `dtype` the type of its rows, `pad` the elements
between the end of a row and the start of the next.
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    embed = dict(op="embed", dtype="bf16", pad=0, world=8, scale=True, absent=0.0)
    grad = dict(op="embed_grad", dtype="bf16", grad_dtype="fp32", pad=0, world=8, scale=True, absent=0.0, one_token=0.0)
    norm = dict(op="norm", dtype="bf16", params="fp32", pad=0, bias=True)
    verify = dict(op="verify", dtype="bf16", pad=0, draft_logits=True, mixed=False, temperature=1.0, agree=0.5, masked=0.0, ragged=False)
    return [
        # the tokens of one decoding step, looked up in the shards of a tied head
        dict(embed, name="embed_decode", n=64, vocab=28672, dim=8192),
        # a long prompt, ids of a padded batch among the tokens, odd width
        dict(embed, name="embed_prompt_odd", n=32771, vocab=50021, dim=4099, dtype="fp16", world=1, scale=False, absent=0.1),
        # one training step's micro-batch, 32-bit main gradients
        dict(grad, name="embed_grad_step", n=65536, vocab=32768, dim=4096),
        # a short batch half of which is one token, gradients in the weights' type, odd width
        dict(grad, name="embed_grad_skewed_odd", n=9001, vocab=16381, dim=2561, grad_dtype="bf16", world=1, one_token=0.5, absent=0.1),
        # the norm in front of the head in a decoding step
        dict(norm, name="norm_decode", rows=64, dim=8192),
        # a long prompt
        dict(norm, name="norm_prompt", rows=32768, dim=4096, params="bf16"),
        # one training step's micro-batch
        dict(norm, name="norm_grad_step", op="norm_grad", rows=16384, dim=4096),
        # rows that start at any element, odd width, weights of the rows' type, no bias
        dict(norm, name="norm_grad_odd", op="norm_grad", rows=5003, dim=2563, dtype="fp16", params="fp16", pad=2, bias=False),
        # one conversation, four drafted tokens
        dict(verify, name="verify_one", sequences=1, drafts=4, vocab=128000),
        # a serving batch with a temperature of its own for each sequence, some of them greedy
        dict(verify, name="verify_batch", sequences=64, drafts=4, vocab=128000, mixed=True),
        # drafts found in the prompt (no logits of their own), of different lengths; grammars mask most tokens; odd width, 32-bit logits
        dict(verify, name="verify_prompt_odd", sequences=100, drafts=7, vocab=50021, dtype="fp32", draft_logits=False, masked=0.9, ragged=True,
             temperature=0.7),
        # a large batch with a small vocabulary
        dict(verify, name="verify_many", sequences=512, drafts=3, vocab=16384),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad", "verify", "verify"])
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, 8, 3]))
    if op == "verify":
        vocab = _log(rng, 4000, 160000)
        case.update(vocab=vocab // 64 * 64 if rng.random() < 0.5 else vocab, drafts=rng.randint(0, 8), draft_logits=rng.random() < 0.6,
                    mixed=rng.random() < 0.4, temperature=rng.choice([1.0, 0.7, 1.5]), agree=rng.choice([0.2, 0.5, 1.0]),
                    masked=rng.choice([0.0, 0.0, 0.9]), ragged=rng.random() < 0.4)
        row = (2 * case["drafts"] + 1) * case["vocab"]
        case["sequences"] = _log(rng, 1, max(1, min(512, 64 * 9 * 128000 // row)))
        return case
    dim = _log(rng, 128, 16384)
    case["dim"] = dim // 64 * 64 if rng.random() < 0.5 else dim
    if op.startswith("norm"):
        case.update(params=rng.choice(["fp32", case["dtype"]]), bias=rng.random() < 0.7)
        case["rows"] = _log(rng, 1, min(65536, 32768 * 4096 * 2 // (case["dim"] * SIZE[case["dtype"]])))
        return case
    case.update(world=rng.choice([1, 2, 8]), scale=rng.random() < 0.5, absent=rng.choice([0.0, 0.2]))
    case["vocab"] = max(8, _log(rng, 1000, min(160000, 32768 * 4096 // case["dim"])) // 8 * 8 if case["dim"] < 16384 else 4096)
    if op == "embed_grad":
        case.update(grad_dtype=rng.choice(["fp32", case["dtype"]]), one_token=rng.choice([0.0, 0.0, 0.3]))
    case["n"] = _log(rng, 1, min(65536, 65536 * 4096 * 2 // (case["dim"] * SIZE[case["dtype"]])))
    return case


def _f32(x):
    """As the calls take it."""
    return float(torch.tensor(x, dtype=torch.float32))


def _rows(rows, dim, pad, dtype):
    return torch.empty(rows, dim + pad, dtype=DTYPE[dtype], device="cuda")[:, :dim]


def _fill(out, gen, make):
    """out <- make(random rows), a part at a time."""
    step = max(1, (1 << 28) // max(1, out.shape[1]))
    for i in range(0, out.shape[0], step):
        part = out[i:i + step]
        part.copy_(make(torch.randn(part.shape, device="cuda", generator=gen)))
    return out


def _prepare_tokens(case, gen):
    """Ids as in text: the k-th most frequent one about as often as 1 / k."""
    n, vocab = case["n"], case["vocab"]
    rank = (torch.rand(n, device="cuda", generator=gen, dtype=torch.float64) * math.log(vocab + 1)).exp().long() - 1
    t = torch.randperm(vocab, device="cuda", generator=gen)[rank.clamp_(0, vocab - 1)]
    if case.get("one_token"):
        t = torch.where(torch.rand(n, device="cuda", generator=gen) < case["one_token"], t[:1], t)
    if case["absent"]:
        t = torch.where(torch.rand(n, device="cuda", generator=gen) < case["absent"], -1, t)
    return t


def _prepare_verify(case, gen, s):
    b, n, vocab = case["sequences"], case["drafts"], case["vocab"]
    z = _rows(b * (n + 1), vocab, case["pad"], case["dtype"])
    at = torch.randint(0, vocab, (b * (n + 1), 32), device="cuda", generator=gen)
    up = torch.rand(at.shape, device="cuda", generator=gen) * 9 + 3
    step = max(1, (1 << 28) // vocab)
    for i in range(0, z.shape[0], step):                # a broad bulk and a few tokens that stand out
        x = torch.randn(z[i:i + step].shape, device="cuda", generator=gen) * 2
        if case["masked"]:
            x.masked_fill_(torch.rand(x.shape, device="cuda", generator=gen) < case["masked"], -math.inf)
        z[i:i + step] = x.scatter_add_(1, at[i:i + step], up[i:i + step])
    scale = torch.full((b,), 1.0 / case["temperature"], device="cuda")
    if case["mixed"]:
        scale = 1 / (torch.rand(b, device="cuda", generator=gen) + 0.5)
        scale[3::4] = math.inf                          # greedy
    s.update(logits=z, scale=_f32(1.0 / case["temperature"]), scales=scale if case["mixed"] else None, draft_logits=None)
    s["uniform"] = torch.rand(b, n, device="cuda", generator=gen)
    s["noise"] = torch.empty(b, vocab, device="cuda").exponential_(generator=gen)
    soft = torch.where(scale.isinf(), 100.0, scale)
    ids = torch.empty(b, n, dtype=torch.int64, device="cuda")
    if case["draft_logits"]:
        s["draft_logits"] = _rows(b * n, vocab, case["pad"], case["dtype"])
    for i in range(b if n else 0):                      # a draft that agrees with the target in part, and tokens drawn from it
        y = z[i * (n + 1):(i + 1) * (n + 1) - 1].float()
        if case["draft_logits"]:
            y = y + torch.randn(y.shape, device="cuda", generator=gen) * case["agree"]
            s["draft_logits"][i * n:(i + 1) * n] = y
            y = s["draft_logits"][i * n:(i + 1) * n].float()
        race = torch.empty_like(y).exponential_(generator=gen)
        ids[i] = (y * soft[i] - race.log()).argmax(1)
    if case["ragged"] and n:
        ids.masked_fill_(torch.arange(n, device="cuda") >= torch.randint(0, n + 1, (b, 1), device="cuda", generator=gen), -1)
    s["draft_ids"] = ids
    s["tokens"] = torch.empty(b, n + 1, dtype=torch.int64, device="cuda")
    s["accepted"] = torch.empty(b, dtype=torch.int64, device="cuda")
    s["logprob"] = torch.empty(b, n + 1, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op == "verify":
        _prepare_verify(case, gen, s)
    elif op.startswith("norm"):
        rows, dim, p = case["rows"], case["dim"], DTYPE[case["params"]]
        spread = torch.exp(torch.randn(dim, device="cuda", generator=gen) * 0.5)
        spread[torch.randint(0, dim, (max(1, dim // 1000),), device="cuda", generator=gen)] *= 30     # a few channels that stand out
        offset = torch.randn(dim, device="cuda", generator=gen) * 0.3
        s["x"] = _fill(_rows(rows, dim, case["pad"], case["dtype"]), gen, lambda x: x * spread + offset)
        s["weight"] = (1 + 0.2 * torch.randn(dim, device="cuda", generator=gen)).to(p)
        s["bias"] = (0.1 * torch.randn(dim, device="cuda", generator=gen)).to(p) if case["bias"] else None
        if op == "norm":
            s["y"], s["stats"] = _rows(rows, dim, case["pad"], case["dtype"]), torch.empty(rows, 2, device="cuda")
        else:
            x = s["x"].float()
            mean = x.mean(1, keepdim=True)
            s["stats"] = torch.cat([mean, (x - mean).square_().mean(1, keepdim=True).add_(1e-5).rsqrt_()], 1)
            s["dy"] = _fill(_rows(rows, dim, case["pad"], case["dtype"]), gen, lambda x: x)
            s["dx"] = _rows(rows, dim, case["pad"], case["dtype"])
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"]) if case["bias"] else None
    else:
        n, vocab, dim, world = case["n"], case["vocab"], case["dim"], case["world"]
        s["tokens"] = _prepare_tokens(case, gen)
        s["scale"] = _f32(math.sqrt(dim)) if case["scale"] else 1.0
        if op == "embed":
            s["table"] = _fill(torch.empty(vocab, dim, dtype=DTYPE[case["dtype"]], device="cuda"), gen, lambda x: x * 0.02)
            s["shards"] = list(s["table"].chunk(world))             # one a rank, as the head's B shards
            s["out"] = _rows(n, dim, case["pad"], case["dtype"])
        else:
            s["grad_out"] = _fill(_rows(n, dim, case["pad"], case["dtype"]), gen, lambda x: x)
            s["grad"] = torch.empty(vocab, dim, dtype=DTYPE[case["grad_dtype"]], device="cuda")
            s["shards"] = list(s["grad"].chunk(world))
    if own:
        import paper_2511_12500_b200 as iris
        need = {"verify": lambda: iris.iris_verify_workspace_bytes(case["sequences"], case["drafts"]),
                "norm_grad": lambda: iris.iris_layer_norm_workspace_bytes(case["rows"], case["dim"]),
                "embed_grad": lambda: iris.iris_embed_workspace_bytes(case["n"], case["vocab"], case["dim"])}.get(op)
        s["workspace"] = torch.empty(need(), dtype=torch.uint8, device="cuda") if need else None
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _plain_embed(s):
    t = s["tokens"]
    y = s["table"][t.clamp_min(0)].float() * s["scale"]
    return {"out": y.masked_fill_((t < 0)[:, None], 0.0).to(s["out"].dtype)}


def _plain_embed_grad(s):
    t = s["tokens"]
    g = (s["grad_out"].float() * s["scale"]).masked_fill_((t < 0)[:, None], 0.0)
    d = torch.zeros(s["grad"].shape, device="cuda").index_add_(0, t.clamp_min(0), g)
    return {"grad": d.to(s["grad"].dtype)}


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    x -= mean
    r = ((x * x).mean(1, keepdim=True) + 1e-5).rsqrt()
    y = x * r * s["weight"].float()
    if s["bias"] is not None:
        y += s["bias"].float()
    return {"y": y.to(s["y"].dtype), "stats": torch.cat([mean, r], 1)}


def _plain_norm_grad(s):
    dy, r = s["dy"].float(), s["stats"][:, 1:]
    xh = (s["x"].float() - s["stats"][:, :1]) * r
    out = {"dweight": (dy * xh).sum(0).to(s["weight"].dtype)}
    if s["bias"] is not None:
        out["dbias"] = dy.sum(0).to(s["weight"].dtype)
    g = dy * s["weight"].float()
    out["dx"] = ((g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * r).to(s["dx"].dtype)
    return out


def _plain_verify(s):
    """In 64 bits: which token it is goes by comparisons."""
    case = s["case"]
    b, n, vocab = case["sequences"], case["drafts"], case["vocab"]
    scale = s["scales"] if s["scales"] is not None else torch.full((b,), s["scale"], device="cuda")
    greedy = scale.isinf()

    def log_probs(rows, each):
        z = rows.double().view(b, each, vocab)
        m = z.amax(2, keepdim=True).clamp_min(-1e300)
        y = (z - m) * torch.where(greedy, 1.0, scale).double()[:, None, None]
        y -= y.exp().sum(2, keepdim=True).log()
        best = torch.zeros_like(y, dtype=torch.bool).scatter_(2, z.argmax(2, keepdim=True), True)
        return torch.where(greedy[:, None, None], torch.where(best, 0.0, -math.inf), y)

    lp, ids = log_probs(s["logits"], n + 1), s["draft_ids"]
    there = (ids >= 0).long().cumprod(1) > 0
    at = ids.clamp_min(0)[:, :, None]
    if n and s["draft_logits"] is not None:
        lq = log_probs(s["draft_logits"], n)
    else:
        lq = torch.full((b, n, vocab), -math.inf, dtype=torch.float64, device="cuda").scatter_(2, at, 0.0)
    ratio = (lp[:, :n].gather(2, at) - torch.where(greedy[:, None, None], 0.0, lq.gather(2, at)))[:, :, 0].exp()
    taken = (there & (s["uniform"].double() < ratio)).long().cumprod(1).sum(1)
    stop = taken[:, None, None].expand(-1, 1, vocab)
    p = lp.gather(1, stop)[:, 0].exp()
    left = p
    if n:
        refused = (taken < n) & there.gather(1, taken.clamp_max(n - 1)[:, None])[:, 0]
        left = (p - torch.where(refused[:, None], lq.gather(1, stop.clamp_max(n - 1))[:, 0].exp(), 0.0)).clamp_min_(0)
        left = torch.where(left.amax(1, keepdim=True) > 0, left, p)
    best = torch.where(greedy, p.argmax(1), (left / s["noise"].double()).argmax(1))
    places = torch.arange(n + 1, device="cuda")
    drafted = torch.cat([ids, ids.new_full((b, 1), -1)], 1)
    tokens = torch.where(places < taken[:, None], drafted, torch.where(places == taken[:, None], best[:, None], -1))
    logprob = torch.where(tokens >= 0, lp.gather(2, tokens.clamp_min(0)[:, :, None])[:, :, 0], 0.0)
    return {"tokens": tokens, "accepted": taken, "logprob": logprob.float()}


PLAIN = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad, "verify": _plain_verify}


# ------------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    import paper_2511_12500_b200 as iris
    case, op = s["case"], s["case"]["op"]
    kind = iris.LOGIT_DTYPES[case["dtype"]]
    if op == "verify":
        stride = case["vocab"] + case["pad"]
        iris.iris_verify_drafts(s["logits"], case["sequences"], case["drafts"], case["vocab"], kind, s["draft_ids"], s["uniform"], s["noise"], s["tokens"],
                                s["accepted"], s["workspace"], draft_logits=s["draft_logits"], logprob=s["logprob"], scale=s["scale"], scales=s["scales"],
                                row_stride=stride, draft_stride=stride)
        return {k: s[k] for k in ("tokens", "accepted", "logprob")}
    stride = case["dim"] + case["pad"]
    if op == "embed":
        iris.iris_embed_tokens(s["shards"], case["vocab"], case["dim"], kind, s["tokens"], case["n"], s["out"], scale=s["scale"], out_stride=stride)
        return {"out": s["out"]}
    if op == "embed_grad":
        iris.iris_embed_tokens_backward(s["grad_out"], case["n"], case["dim"], kind, s["tokens"], s["shards"], case["vocab"],
                                        iris.LOGIT_DTYPES[case["grad_dtype"]], s["workspace"], scale=s["scale"], grad_out_stride=stride)
        return {"grad": s["grad"]}
    params = iris.LOGIT_DTYPES[case["params"]]
    if op == "norm":
        iris.iris_layer_norm(s["x"], case["rows"], case["dim"], kind, s["y"], weight=s["weight"], bias=s["bias"], param_dtype=params, stats=s["stats"],
                             eps=1e-5, row_stride=stride, out_stride=stride)
        return {"y": s["y"], "stats": s["stats"]}
    iris.iris_layer_norm_backward(s["x"], case["rows"], case["dim"], kind, s["dy"], s["stats"], s["workspace"], weight=s["weight"], param_dtype=params,
                                  dx=s["dx"], dweight=s["dweight"], dbias=s["dbias"], row_stride=stride, dy_stride=stride, dx_stride=stride)
    return {k: s[k] for k in ("dweight", "dbias", "dx") if s[k] is not None}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_embed(case, s):
    t = s["tokens"]
    out = torch.zeros(case["n"], case["dim"], dtype=torch.float64, device="cuda")
    here = torch.nonzero(t >= 0)[:, 0]
    out[here] = s["scale"] * s["table"].double()[t[here]]
    return {"out": out}


def _exact_embed_grad(case, s):
    order = torch.argsort(s["tokens"], stable=True)
    order = order[s["tokens"][order] >= 0]
    ids, counts = torch.unique_consecutive(s["tokens"][order], return_counts=True)
    out = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
    for a in range(0, case["dim"], 512):
        out[ids, a:a + 512] = s["scale"] * torch.segment_reduce(s["grad_out"][:, a:a + 512].double()[order], "sum", lengths=counts)
    return {"grad": out}


def _exact_norm(case, s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    y = (x - mean) / (var + 1e-5).sqrt() * s["weight"].double()
    if s["bias"] is not None:
        y = y + s["bias"].double()
    return {"y": y, "stats": torch.cat([mean, 1 / (var + 1e-5).sqrt()], 1)}


def _exact_norm_grad(case, s):
    dy, x, mean, r = s["dy"].double(), s["x"].double(), s["stats"][:, :1].double(), s["stats"][:, 1:].double()
    dim, w = case["dim"], s["weight"].double()
    out = {"dweight": torch.einsum("rj,rj->j", dy * r, x) - torch.einsum("rj,r->j", dy, (mean * r)[:, 0])}
    if s["bias"] is not None:
        out["dbias"] = dy.sum(0)
    along = (torch.mv(dy * x, w)[:, None] - mean * torch.mv(dy, w)[:, None]) * r / dim
    out["dx"] = r * (dy * w - torch.mv(dy, w)[:, None] / dim - (x - mean) * r * along)
    return out


def _exact_verify(case, s):
    """The log probabilities of the tokens that the plain form names; whole numbers are compared with the plain form's."""
    b, n, vocab = case["sequences"], case["drafts"], case["vocab"]
    tokens = _plain_verify(s)["tokens"]
    out = torch.zeros(b, n + 1, dtype=torch.float64, device="cuda")
    for i in range(b):
        scale = float(s["scales"][i]) if s["scales"] is not None else s["scale"]
        if not math.isinf(scale):                       # a greedy sequence's tokens are certain
            lp = torch.log_softmax(s["logits"][i * (n + 1):(i + 1) * (n + 1)].double() * scale, 1)
            out[i] = torch.where(tokens[i] >= 0, lp.gather(1, tokens[i].clamp_min(0)[:, None])[:, 0], 0.0)
    return {"tokens": None, "accepted": None, "logprob": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "norm": _exact_norm, "norm_grad": _exact_norm_grad,
            "verify": _exact_verify}[case["op"]](case, s)


def _distinct(case):
    """How many different ids the tokens have on average."""
    vocab, n = case["vocab"], case["n"] * (1 - case["absent"])
    k = torch.arange(vocab, dtype=torch.float64)
    p = (torch.log(k + 2) - torch.log(k + 1)) / math.log(vocab + 1)
    return int((1 - (1 - p) ** n).sum())


def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "verify":
        b, n, vocab = case["sequences"], case["drafts"], case["vocab"]
        rows = b * (n + 1 + n * case["draft_logits"])
        return {"bytes": rows * vocab * size + b * vocab * 4 + b * (n + 1) * 24, "flops": rows * vocab * 4 + b * vocab * 8}
    dim = case["dim"]
    if op.startswith("norm"):
        cells, p = case["rows"] * dim, SIZE[case["params"]] * dim
        back = op == "norm_grad"
        return {"bytes": cells * size * (3 if back else 2) + p * (2 + 2 * back), "flops": cells * (14 if back else 8)}
    cells = case["n"] * dim
    if op == "embed":
        return {"bytes": (cells + _distinct(case) * dim) * size + case["n"] * 8, "flops": cells}
    return {"bytes": cells * size + case["vocab"] * dim * SIZE[case["grad_dtype"]] + case["n"] * 8, "flops": cells}
