"""Cases for the operators on logits: token log probabilities (forward and backward) and distillation from a teacher's top logits.

Each case is one call as a serving loop, an evaluation or a training step makes it on the logits of a head: `op` says which operator,
`rows` x `vocab` the logits, `dtype` their type, `pad` the elements between the end of a row and the start of the next.
"""
import math

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
LOWEST = torch.finfo(torch.float32).min


def listed():
    score = dict(op="score", dtype="bf16", pad=0, targets=1, top=0, entropy=True, masked=0.0, temperature=1.0)
    grad = dict(op="score_grad", dtype="bf16", pad=0, targets=1, entropy=True, temperature=1.0)
    step = dict(op="distill_step", dtype="bf16", pad=0, k=64, tail=False, temperature=1.0, unused=0)
    return [
        # one sequence being decoded: the sampled token's log probability and five alternatives, where latency is all
        dict(score, name="score_decode_1", rows=1, vocab=16384, top=5),
        # a decoding batch with a large vocabulary, twenty alternatives, a sampling temperature
        dict(score, name="score_decode_64", rows=64, vocab=128000, top=20, temperature=0.7),
        # constrained decoding: a grammar leaves a few tokens of each row, one row nothing; odd width, 32-bit logits
        dict(score, name="score_masked_odd", rows=333, vocab=50021, dtype="fp32", top=10, masked=0.998),
        # log probabilities of a long prompt
        dict(score, name="score_prompt", rows=4096, vocab=128000),
        # a teacher's list for distillation
        dict(score, name="score_teacher", rows=4096, vocab=36864, dtype="fp16", top=64, targets=0, entropy=False),
        # policy gradient with an entropy bonus
        dict(grad, name="score_grad", rows=8192, vocab=16384),
        # several answers scored at one position, odd width, rows that start at any element
        dict(grad, name="score_grad_odd", rows=700, vocab=50021, dtype="fp16", targets=4, entropy=False, temperature=1.3),
        # distillation of a few positions
        dict(step, name="distill_small", rows=16, vocab=16384, k=16),
        # one training step's micro-batch
        dict(step, name="distill_step", rows=8192, vocab=28672, temperature=2.0),
        # large vocabulary with padded columns, teacher's log probabilities with the remainder as one more token
        dict(step, name="distill_step_tail", rows=4096, vocab=128000, tail=True, unused=256),
        # evaluation: the loss alone, 32-bit logits, odd width
        dict(step, name="distill_eval", op="distill_loss", rows=1024, vocab=50021, dtype="fp32", k=100, tail=True),
        # the gradient from statistics of an earlier forward pass
        dict(step, name="distill_grad", op="distill_grad", rows=2048, vocab=36864, dtype="fp16", pad=8, k=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "score", "score_grad", "distill_step", "distill_step", "distill_loss", "distill_grad"])
    vocab = _log(rng, 4000, 160000)
    if rng.random() < 0.5:
        vocab = vocab // 64 * 64
    case = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), pad=rng.choice([0, 0, 0, 8, 3]), vocab=vocab)
    case["rows"] = _log(rng, 1, min(8192, 4096 * 128000 // (vocab * SIZE[case["dtype"]] // 2)))
    case["temperature"] = rng.choice([1.0, 1.0, 0.7, 2.0])
    if op.startswith("score"):
        case.update(targets=rng.choice([1, 1, 1, 4]), entropy=rng.random() < 0.7)
    else:
        case.update(k=_log(rng, 1, 128), tail=rng.random() < 0.5, unused=rng.choice([0, 0, 100]))
    if op == "score":
        case.update(top=rng.choice([0, _log(rng, 1, 128)]), masked=rng.choice([0.0, 0.0, 0.25, 0.998]))
    return case


def _logits(case, gen, boost=32):
    """Rows as a trained head gives them: a broad bulk and a few tokens that stand out."""
    rows, vocab = case["rows"], case["vocab"]
    store = torch.empty(rows, vocab + case["pad"], dtype=DTYPE[case["dtype"]], device="cuda")
    at = torch.randint(0, vocab, (rows, boost), device="cuda", generator=gen)
    up = torch.rand(rows, boost, device="cuda", generator=gen) * 9 + 3
    step = max(1, (1 << 28) // max(1, vocab))
    for i in range(0, rows, step):
        x = torch.randn(min(step, rows - i), vocab + case["pad"], device="cuda", generator=gen) * 2.5
        x.scatter_add_(1, at[i:i + step], up[i:i + step])
        store[i:i + step] = x
    return store[:, :vocab], at


def _statistics(z, scale):
    """Per row: the largest logit and ln sum exp(scale (z - largest)), as the forward call leaves them."""
    m = z.float().amax(-1, keepdim=True).clamp_min(LOWEST)
    return m, ((z.float() - m) * scale).exp().sum(-1, keepdim=True).log()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, rows, vocab = case["op"], case["rows"], case["vocab"]
    z, at = _logits(case, gen)
    s = {"case": case, "logits": z, "scale": 1.0 / case["temperature"]}
    f32 = dict(dtype=torch.float32, device="cuda")
    if op.startswith("score"):
        q = case["targets"]
        t = torch.cat([at[:, :1], torch.randint(0, vocab, (rows, 3), device="cuda", generator=gen)], 1)[:, :q].contiguous()
        t[5::16] = -1                                       # padding positions
        s["targets"] = t
    if op == "score":
        if case["masked"]:
            step = max(1, (1 << 28) // vocab)
            for i in range(0, rows, step):
                gone = torch.rand(min(step, rows - i), vocab, device="cuda", generator=gen) < case["masked"]
                z[i:i + step].masked_fill_(gone, -math.inf)
            if rows > 2:
                z[rows // 2] = -math.inf                    # a row that its mask leaves empty
        s["logprob"] = torch.empty(rows, case["targets"], **f32)
        s["entropy"] = torch.empty(rows, **f32) if case["entropy"] else None
        s["stats"] = torch.empty(rows, 2, **f32)
        s["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int64, device="cuda") if case["top"] else None
        s["top_logprob"] = torch.empty(rows, case["top"], **f32) if case["top"] else None
    elif op == "score_grad":
        m, ls = _statistics(z, s["scale"])
        s["stats"] = torch.cat([m, ls], 1)
        s["grad_logprob"] = torch.randn(rows, case["targets"], device="cuda", generator=gen)
        s["grad_entropy"] = s["entropy"] = None
        if case["entropy"]:
            d = ((z.float() - m) * s["scale"]).clamp_min(-1e4)
            s["entropy"] = ls[:, 0] - (d.exp() * d).sum(-1) / ls[:, 0].exp()
            s["grad_entropy"] = torch.rand(rows, device="cuda", generator=gen) * 0.01
            del d
    else:
        if case["unused"]:
            z[:, vocab - case["unused"]:] = -math.inf       # columns that pad the vocabulary
        k = min(case["k"], vocab)
        s["teacher"], s["ids"] = torch.empty(rows, k, **f32), torch.empty(rows, k, dtype=torch.int64, device="cuda")
        step = max(1, (1 << 27) // vocab)
        for i in range(0, rows, step):                      # a teacher that agrees with the student in part
            y = z[i:i + step].float()
            y = y + torch.randn(y.shape, device="cuda", generator=gen)
            v, s["ids"][i:i + step] = y.topk(k, dim=-1)
            s["teacher"][i:i + step] = v - torch.logsumexp(y, -1, keepdim=True) if case["tail"] else v
        if k > 4:
            s["ids"][3::7, -2:] = -1                        # shorter lists
        s["weight"] = (torch.rand(rows, device="cuda", generator=gen) + 0.5) * (64.0 if case["dtype"] == "fp16" else 1.0)
        s["weight"][5::16] = 0                              # padding positions
        s["loss"] = torch.empty(rows, **f32)
        s["stats"] = torch.empty(rows, 3, **f32)
        if op == "distill_grad":
            m, ls = _statistics(z, s["scale"])
            rest = torch.zeros_like(ls)
            if case["tail"]:
                rest = _tail(((z.float() - m) * s["scale"]).exp(), s["ids"]).sum(-1, keepdim=True).log()
            s["stats"] = torch.cat([m, ls, rest], 1)
    if op in ("score_grad", "distill_step", "distill_grad"):
        s["dlogits"] = torch.empty(rows, vocab + case["pad"], dtype=z.dtype, device="cuda")[:, :vocab]
    torch.cuda.synchronize()
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _tail(e, ids):
    """e with 0 for the tokens on the list."""
    there = ids >= 0
    listed = torch.zeros_like(e, dtype=torch.bool).scatter_(1, ids.clamp_min(0), there)
    listed[:, :1] = ((ids == 0) & there).any(1, keepdim=True)
    return e.masked_fill(listed, 0.0)


def _top(x, k):
    """The k largest of each row in order, the lowest index first among equals: one 64-bit key a column."""
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (order << 32) + (0xFFFFFFFF - torch.arange(x.shape[1], device=x.device))
    return 0xFFFFFFFF - (key.topk(k, dim=-1).values & 0xFFFFFFFF)


def _plain_score(s):
    case, scale, t = s["case"], s["scale"], s["targets"]
    x = s["logits"].float()
    m = x.amax(-1, keepdim=True).clamp_min(LOWEST)
    d = (x - m) * scale
    e = d.exp()
    total = e.sum(-1, keepdim=True)
    ls = total.log()
    some = total > 0

    def logprob(ids):
        return torch.where(some, d.gather(1, ids) - ls, -math.inf)

    out = {"stats": torch.cat([torch.where(some, m, -math.inf), ls], 1), "logprob": torch.where(t < 0, 0.0, logprob(t.clamp_min(0)))}
    if case["entropy"]:
        mean = (e * d.clamp_min(-1e4)).sum(-1, keepdim=True) / total
        out["entropy"] = torch.where(some, ls - mean, 0.0)[:, 0]
    if case["top"]:
        out["top_ids"] = _top(x, case["top"])
        out["top_logprob"] = logprob(out["top_ids"])
    return out


def _plain_score_grad(s):
    z, t, g, scale = s["logits"], s["targets"], s["grad_logprob"], s["scale"]
    m, ls = s["stats"][:, :1], s["stats"][:, 1:]
    lq = (z.float() - m) * scale - ls
    q = lq.exp()
    g = torch.where(t < 0, 0.0, g)
    dz = -g.sum(1, keepdim=True) * q
    if s["grad_entropy"] is not None:
        dz -= s["grad_entropy"][:, None] * q * (lq.clamp_min(-1e4) + s["entropy"][:, None])
    dz.scatter_add_(1, t.clamp_min(0), g)
    return {"dlogits": (dz * scale).to(z.dtype)}


def _teacher(s):
    """The teacher's probabilities of the listed tokens and of the remainder."""
    v, there = s["teacher"], s["ids"] >= 0
    if s["case"]["tail"]:
        p = torch.where(there, v.exp(), 0.0)
        return p, (1 - p.sum(1, keepdim=True)).clamp_min(0)
    v = torch.where(there, v * s["scale"], -math.inf)
    e = (v - v.amax(1, keepdim=True).clamp_min(LOWEST)).exp()
    return e / e.sum(1, keepdim=True).clamp_min(1e-30), torch.zeros_like(e[:, :1])


def _xlogy(p, lq):
    """p (ln p - lq), 0 where p is 0."""
    return torch.where(p > 0, p * (p.clamp_min(1e-45).log() - lq), 0.0)


def _plain_distill(s):
    case, z, ids, scale = s["case"], s["logits"], s["ids"], s["scale"]
    p, rest = _teacher(s)
    out = {}
    x = z.float()
    saved = case["op"] == "distill_grad"
    m = s["stats"][:, :1] if saved else x.amax(-1, keepdim=True)
    d = (x - m) * scale
    e = d.exp()
    tail = _tail(e, ids) if case["tail"] else None
    if saved:
        ls, lr = s["stats"][:, 1:2], s["stats"][:, 2:]
    else:
        ls = e.sum(-1, keepdim=True).log()
        lr = tail.sum(1, keepdim=True).log() if case["tail"] else torch.zeros_like(ls)
        loss = _xlogy(p, d.gather(1, ids.clamp_min(0)) - ls).sum(1)
        if case["tail"]:
            loss += _xlogy(rest, lr - ls)[:, 0]
        out = {"stats": torch.cat([m, ls, lr], 1), "loss": loss}
    if case["op"] != "distill_loss":
        dz = e * ((p.sum(1, keepdim=True) + rest) / ls.exp())
        if case["tail"]:
            dz -= tail * (rest / lr.exp())
        dz.scatter_add_(1, ids.clamp_min(0), -p)
        out["dlogits"] = (dz * (s["weight"][:, None] * scale)).to(z.dtype)
    return out


# ------------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    import paper_2511_12500_b200 as iris
    case, z, op = s["case"], s["logits"], s["case"]["op"]
    where = (z, case["rows"], case["vocab"], iris.LOGIT_DTYPES[case["dtype"]])
    stride = case["vocab"] + case["pad"]
    if op == "score":
        iris.iris_token_logprobs(*where, targets=s["targets"], n_targets=case["targets"], logprob=s["logprob"], entropy=s["entropy"],
                                 stats=s["stats"], top_k=case["top"], top_ids=s["top_ids"], top_logprob=s["top_logprob"],
                                 scale=s["scale"], row_stride=stride)
        return {k: s[k] for k in ("stats", "logprob", "entropy", "top_ids", "top_logprob") if s[k] is not None}
    if op == "score_grad":
        iris.iris_token_logprobs_backward(*where, s["targets"], case["targets"], s["stats"], s["grad_logprob"], s["dlogits"],
                                          entropy=s["entropy"], grad_entropy=s["grad_entropy"], scale=s["scale"], row_stride=stride,
                                          grad_stride=stride)
        return {"dlogits": s["dlogits"]}
    mode = iris.IRIS_DISTILL_TAIL if case["tail"] else iris.IRIS_DISTILL_RENORM
    k = s["ids"].shape[1]
    if op == "distill_grad":
        iris.iris_distill_topk_backward(*where, s["teacher"], s["ids"], k, s["stats"], s["weight"], s["dlogits"], mode=mode,
                                        scale=s["scale"], teacher_scale=s["scale"], row_stride=stride, grad_stride=stride)
        return {"dlogits": s["dlogits"]}
    step = op == "distill_step"
    iris.iris_distill_topk(*where, s["teacher"], s["ids"], k, s["loss"], mode=mode, stats=s["stats"], weight=s["weight"] if step else None,
                           dlogits=s["dlogits"] if step else None, scale=s["scale"], teacher_scale=s["scale"], row_stride=stride,
                           grad_stride=stride)
    return {"stats": s["stats"], "loss": s["loss"], **({"dlogits": s["dlogits"]} if step else {})}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_score(state) if op == "score" else _plain_score_grad(state) if op == "score_grad" else _plain_distill(state)


# ------------------------------------------------------------------------------------------------- 64 bits
def _exact_rows(case, s, a, b):
    """The definition for rows a..b in 64 bits."""
    z = s["logits"][a:b].double()
    c, n = s["scale"], z.shape[1]
    lse = torch.logsumexp(c * z, 1, keepdim=True)
    empty = torch.isneginf(lse)
    lq = torch.where(empty, -math.inf, c * z - torch.where(empty, 0.0, lse))
    m = z.max(1, keepdim=True).values
    ls = torch.where(empty, -math.inf, lse - c * torch.where(empty, 0.0, m))
    q = lq.exp()
    op = case["op"]
    if op == "score":
        t = s["targets"][a:b]
        out = {"stats": torch.cat([m, ls], 1), "logprob": torch.where(t < 0, 0.0, lq.gather(1, t.clamp(min=0)))}
        if case["entropy"]:
            out["entropy"] = -(q * torch.where(q > 0, lq, 0.0)).sum(1)
        if case["top"]:
            best = lq.topk(case["top"], 1).values             # values are unique even where places are not
            out["top_ids"], out["top_logprob"] = None, best
        return out
    if op == "score_grad":
        t, g = s["targets"][a:b], s["grad_logprob"][a:b].double()
        dz = torch.zeros_like(z)
        g = g.masked_fill(t < 0, 0.0)
        dz.scatter_add_(1, t.clamp(min=0), g)
        dz -= g.sum(1, keepdim=True) * q
        if s["grad_entropy"] is not None:
            h = -(q * torch.where(q > 0, lq, 0.0)).sum(1, keepdim=True)
            dz -= s["grad_entropy"][a:b, None].double() * q * (torch.where(q > 0, lq, 0.0) + h)
        return {"dlogits": c * dz}
    ids, v = s["ids"][a:b], s["teacher"][a:b].double()
    there = ids >= 0
    target = torch.zeros(z.shape[0], n + 1, dtype=torch.float64, device=z.device)   # one more column takes what is absent
    where = torch.where(there, ids, n)
    p = torch.where(there, v.exp(), 0.0) if case["tail"] else torch.softmax(torch.where(there, c * v, -math.inf), 1)
    target.scatter_(1, where, p)
    target = target[:, :n]
    mark = torch.zeros(z.shape[0], n + 1, dtype=torch.bool, device=z.device).scatter_(1, where, True)[:, :n]
    loss = torch.where(target > 0, target * (target.log() - lq), 0.0).sum(1)
    dz = target.sum(1, keepdim=True) * q - target
    lr = torch.zeros_like(ls)
    if case["tail"]:
        rest = (1 - target.sum(1, keepdim=True)).clamp(min=0)
        out_q = torch.where(mark, 0.0, q)
        qr = out_q.sum(1, keepdim=True)
        loss += torch.where(rest > 0, rest * (rest.log() - qr.log()), 0.0)[:, 0]
        dz += rest * (q - out_q / qr)
        lr = qr.log() + ls
    out = {}
    if op != "distill_grad":
        out.update(stats=torch.cat([m, ls, lr], 1), loss=loss)
    if op != "distill_loss":
        out["dlogits"] = c * s["weight"][a:b, None].double() * dz
    return out


def exact(case, seed):
    s = prepare(case, seed)
    step = max(1, (1 << 26) // case["vocab"])
    parts = [_exact_rows(case, s, a, min(case["rows"], a + step)) for a in range(0, case["rows"], step)]
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}


def work(case):
    op, rows, cells = case["op"], case["rows"], case["rows"] * case["vocab"]
    grad = op in ("score_grad", "distill_step", "distill_grad")
    small = rows * 8
    if op == "score":
        small += rows * (12 * case["targets"] + 4 * case["entropy"] + 12 * case["top"])
    elif op == "score_grad":
        small += rows * (12 * case["targets"] + 8 * case["entropy"])
    else:
        small += rows * (12 * case["k"] + 12)
    flops = {"score": 5 + 2 * bool(case.get("entropy")), "score_grad": 4 + 3 * bool(case.get("entropy")), "distill_step": 8, "distill_loss": 5,
             "distill_grad": 4}[op]
    return {"bytes": cells * SIZE[case["dtype"]] * (1 + grad) + small, "flops": cells * flops}
