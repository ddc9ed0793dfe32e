"""Operators on logits against their definitions in 64 bits: types, ragged and strided rows, masks, ties, long rows, streams.

Tolerances (set from the arithmetic, 32-bit sums of at most a few hundred terms a thread):
  - largest logit and alternatives' columns: exact;
  - ln sum and log probabilities: 1e-5 + 1e-6 |value|: exponents carry 3 roundings of 2^-24 relative, weighted by probability (< 1e-6 together),
    2^x two units of 2^-23, a thread's sum of n terms n 2^-24 (< 7e-6 up to n = 100);
  - entropy: 3e-5 + 1e-6 |value| (the same for sum y 2^y, whose terms are up to 20 times larger and carry small weights);
  - gradient, by place: half a unit of the stored type + 3e-5 of the sum of the sizes of its terms (2^y for |y| <= 120 carries 120 * 2^-23);
  - loss: 1e-5 + 1e-5 of the sum of the sizes of its terms.
"""
import math

import numpy as np
import pytest
import torch

import logit_ref as ref
import paper_2511_12500_b200 as iris

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
HALF_UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
SMALLEST = {"bf16": 1e-37, "fp16": 2.0 ** -25, "fp32": 1e-37}
SENTINEL = 7.0


def strided(values: np.ndarray, dtype: str, pad: int = 0, offset: int = 0):
    """values [rows, vocab] on the GPU with `pad` elements between rows, starting `offset` elements into an allocation."""
    rows, vocab = values.shape
    store = torch.full((offset + rows * (vocab + pad) + 32,), SENTINEL, dtype=TORCH[dtype], device="cuda")
    view = store[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(torch.from_numpy(values.astype(np.float32)))
    return store, view


def as64(t: torch.Tensor) -> np.ndarray:
    return t.double().cpu().numpy()


def outside_untouched(store, view, offset):
    keep = torch.ones(store.numel(), dtype=torch.bool, device="cuda")
    rows, vocab = view.shape
    if rows and vocab:
        keep[offset:offset + rows * view.stride(0)].view(rows, -1)[:, :vocab] = False
    assert bool((store[keep] == SENTINEL).all())


def logits_like(rng, rows, vocab):
    z = rng.normal(0, 2.5, (rows, vocab))
    z[:, rng.integers(0, max(1, vocab), 3)] += 5 if vocab else 0
    return z


def score(z, dtype, targets=None, top=0, entropy=True, scale=1.0, stride=0, stream=None):
    rows, vocab = z.shape
    f = dict(dtype=torch.float32, device="cuda")
    nt = 0 if targets is None else targets.shape[1]
    out = dict(logprob=torch.full((rows, nt), SENTINEL, **f), entropy=torch.full((rows,), SENTINEL, **f) if entropy else None,
               stats=torch.full((rows, 2), SENTINEL, **f), top_ids=torch.full((rows, top), -7, dtype=torch.int64, device="cuda"),
               top_logprob=torch.full((rows, top), SENTINEL, **f))
    iris.iris_token_logprobs(z, rows, vocab, iris.LOGIT_DTYPES[dtype], targets=targets, n_targets=nt, top_k=top, scale=scale,
                             row_stride=stride or (z.stride(0) if rows > 1 else 0), stream=stream, **out)
    return out


def close(got, want, tol, what):
    got, want, tol = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64), np.broadcast_to(tol, np.shape(want))
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), (what, got[~fine][:5], want[~fine][:5])
    off = np.abs(got[fine] - want[fine])
    assert np.all(off <= tol[fine]), (what, float(np.max(off - tol[fine])), float(off.max()))


def check_score(z, out, targets, top, scale):
    v = as64(z)
    ids, tlp = out["top_ids"].cpu().numpy(), as64(out["top_logprob"])
    for r in range(v.shape[0]):
        m, ls, lq = ref.log_softmax(v[r], scale)
        close(out["stats"][r, 0].item(), m, 0.0, "max")
        close(out["stats"][r, 1].item(), ls, 1e-5, "ln sum")
        if out["entropy"] is not None:
            h = ref.entropy(lq)
            close(out["entropy"][r].item(), h, 3e-5 + 1e-6 * abs(h), "entropy")
        if targets is not None:
            t = targets[r].cpu().numpy()
            want = np.array([lq[j] if 0 <= j < v.shape[1] else 0.0 for j in t])
            close(as64(out["logprob"][r]), want, 1e-5 + 1e-6 * np.abs(want), "logprob")
        if top:
            want = ref.top(v[r], top)
            assert np.array_equal(ids[r], want), (r, ids[r][:8], want[:8])
            close(tlp[r], lq[want], 1e-5 + 1e-6 * np.abs(lq[want]), "top_logprob")


# ------------------------------------------------------------------------------------------------ forward
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,vocab,pad,offset,top,scale", [
    (1, 1, 0, 0, 1, 1.0), (3, 2, 1, 1, 2, 0.5), (5, 7, 0, 0, 3, 1.0), (4, 8, 0, 0, 8, 1.0), (4, 9, 0, 3, 5, 1.0), (2, 31, 2, 5, 31, 2.0),
    (3, 128, 0, 0, 128, 1.0), (7, 1000, 0, 0, 20, 1.0 / 0.7), (3, 1001, 0, 1, 64, 1.0), (2, 4096, 8, 0, 128, 1.0), (3, 4097, 3, 2, 5, 1.0),
    (2, 8200, 0, 7, 1, 1.0), (2, 16384, 0, 0, 20, 1.0), (1, 36864, 0, 0, 64, 1.0), (2, 50021, 0, 0, 33, 1.0), (1, 131072, 0, 0, 20, 0.8),
    (1, 140001, 0, 3, 128, 1.0), (300, 600, 0, 0, 4, 1.0), (9, 2048, 0, 0, 0, 1.0),
])
def test_forward(dtype, rows, vocab, pad, offset, top, scale):
    rng = np.random.default_rng(rows * 7919 + vocab)
    store, z = strided(logits_like(rng, rows, vocab), dtype, pad, offset)
    t = torch.from_numpy(rng.integers(0, vocab, (rows, 3))).cuda()
    t[0, 1] = -1
    t[-1, 2] = vocab
    out = score(z, dtype, t, top, True, scale)
    check_score(z, out, t, top, scale)
    outside_untouched(store, z, offset)


MASKS = ["most", "all", "one", "lowest", "all_lowest", "lowest_and_one", "prefix", "suffix", "inf", "nan", "minus_zero"]


def masked(rng, kind, rows, vocab, dtype):
    z = logits_like(rng, rows, vocab)
    low = float(torch.finfo(TORCH[dtype]).min)
    r = rows // 2
    if kind == "most":
        z[rng.random(z.shape) < 0.99] = -np.inf
    elif kind == "all":
        z[r] = -np.inf
    elif kind == "one":
        z[r] = -np.inf
        z[r, vocab // 3] = 1.5
    elif kind == "lowest":
        z[rng.random(z.shape) < 0.995] = low
    elif kind == "all_lowest":
        z[r] = low
    elif kind == "lowest_and_one":
        z[r] = low
        z[r, vocab - 1] = -3.0
    elif kind == "prefix":
        z[:, :vocab * 2 // 3] = -np.inf
    elif kind == "suffix":
        z[:, vocab // 3:] = low
    elif kind == "inf":
        z[r, vocab // 2] = np.inf
    elif kind == "nan":
        z[r, [1, vocab // 2]] = np.nan
        z[r, 2] = np.inf
    elif kind == "minus_zero":
        z[:] = -0.0
        z[:, ::2] = 0.0
    return z


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [37, 3001, 20000])
@pytest.mark.parametrize("kind", MASKS)
def test_forward_masks(dtype, vocab, kind):
    rng = np.random.default_rng(11)
    _, z = strided(masked(rng, kind, 3, vocab, dtype), dtype, 0, 1)
    t = torch.from_numpy(rng.integers(0, vocab, (3, 2))).cuda()
    t[1, 0] = vocab // 3
    out = score(z, dtype, t, 24, True, 1.0)
    check_score(z, out, t, 24, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["constant", "two_values", "rising", "falling", "steps", "late_peak", "every_64th", "block", "wave"])
@pytest.mark.parametrize("vocab,top", [(5000, 5), (20000, 128), (70000, 40), (140000, 128)])
def test_alternatives_where_many_are_equal_or_in_order(dtype, kind, vocab, top):
    j = np.arange(vocab)
    z = {"constant": 0.25 + 0 * j, "two_values": (j % 3 == 0) * 1.0, "rising": j * 1e-3, "falling": -j * 1e-3, "steps": j // 1000 * 0.5,
         "late_peak": (j >= vocab - top // 2) * 3.0, "every_64th": np.where(j % 64 == 5, 4.0 + j * 1e-5, 0.0), "block": np.where(j // 8 % 256 == 3, 2.0, -j * 1e-6),
         "wave": np.sin(j * 0.01)}[kind]
    _, g = strided(np.stack([z, z[::-1]]), dtype)
    check_score(g, score(g, dtype, None, top), None, top, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("seed", range(6))
def test_alternatives_of_random_rows(dtype, seed):
    rng = np.random.default_rng(seed)
    vocab, top, rows = int(rng.integers(200, 60000)), int(rng.integers(1, 129)), 3
    z = rng.normal(0, 1, (rows, vocab)) if seed % 2 else rng.integers(0, 40, (rows, vocab)).astype(float)
    _, g = strided(z, dtype, int(rng.integers(0, 9)))
    check_score(g, score(g, dtype, None, top), None, top, 1.0)


def test_each_output_may_be_left_out():
    rng = np.random.default_rng(3)
    _, z = strided(logits_like(rng, 4, 900), "bf16")
    t = torch.from_numpy(rng.integers(0, 900, (4, 1))).cuda()
    full = score(z, "bf16", t, 7)
    lone = torch.zeros(4, device="cuda")
    iris.iris_token_logprobs(z, 4, 900, iris.IRIS_BF16, entropy=lone)
    close(as64(lone), as64(full["entropy"]), 1e-5, "entropy alone")   # another variant may sum in another order
    ids = torch.zeros(4, 7, dtype=torch.int64, device="cuda")
    iris.iris_token_logprobs(z, 4, 900, iris.IRIS_BF16, top_k=7, top_ids=ids)
    assert torch.equal(ids, full["top_ids"])
    lp = torch.zeros(4, 1, device="cuda")
    iris.iris_token_logprobs(z, 4, 900, iris.IRIS_BF16, targets=t, n_targets=1, logprob=lp)
    close(as64(lp), as64(full["logprob"]), 1e-5, "logprob alone")


def test_128_targets_and_a_second_run_gives_the_same_bits():
    rng = np.random.default_rng(4)
    _, z = strided(logits_like(rng, 2, 3000), "bf16")
    t = torch.from_numpy(rng.integers(-2, 3002, (2, 128))).cuda()
    a, b = score(z, "bf16", t, 128), score(z, "bf16", t, 128)
    check_score(z, a, t, 128, 1.0)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_rows_beyond_four_gigabytes():
    vocab, stride = 1003, 1_400_000_003
    store = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")    # 5.6 GB
    rng = np.random.default_rng(5)
    values = logits_like(rng, 3, vocab)
    for r in range(3):
        store[r * stride:r * stride + vocab].copy_(torch.from_numpy(values[r].astype(np.float32)))
    z = store.as_strided((3, vocab), (stride, 1))
    t = torch.from_numpy(rng.integers(0, vocab, (3, 1))).cuda()
    out = score(z, "bf16", t, 9)
    check_score(z.clone(), out, t, 9, 1.0)
    g = torch.ones(3, 1, device="cuda")
    iris.iris_token_logprobs_backward(store, 3, vocab, iris.IRIS_BF16, t, 1, out["stats"], g, store, row_stride=stride, grad_stride=stride)
    for r in range(3):
        lq = ref.log_softmax(values[r].astype(np.float32).astype(np.float64), 1.0)[2]
        got = as64(store[r * stride:r * stride + vocab])
        want = -np.exp(lq)
        want[t[r, 0].item()] += 1
        assert np.abs(got - want).max() < 0.02


def test_other_stream_and_no_rows():
    rng = np.random.default_rng(6)
    _, z = strided(logits_like(rng, 64, 9000), "bf16")
    want = score(z, "bf16", None, 12)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    copy = torch.empty_like(z)
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        copy.copy_(z)                       # the call has to come after this on its stream
        got = score(copy, "bf16", None, 12)
    s.synchronize()
    assert torch.equal(got["top_ids"], want["top_ids"]) and torch.equal(got["stats"], want["stats"])
    empty = torch.empty(0, 10, dtype=torch.bfloat16, device="cuda")
    iris.iris_token_logprobs(empty, 0, 10, iris.IRIS_BF16, top_k=3, top_ids=torch.empty(0, 3, dtype=torch.int64, device="cuda"))
    out = score(torch.empty(2, 0, dtype=torch.float32, device="cuda"), "fp32", torch.zeros(2, 1, dtype=torch.int64, device="cuda"))
    assert out["entropy"].tolist() == [0, 0] and out["logprob"].tolist() == [[0], [0]] and bool(torch.isneginf(out["stats"]).all())


# ------------------------------------------------------------------------------------------------ gradient of the forward call
def run_score_grad(z, dtype, t, g, gh, scale, dz, stats=None, entropy=None):
    rows, vocab = z.shape
    if stats is None:
        out = score(z, dtype, None, 0, True, scale)
        stats, entropy = out["stats"], out["entropy"]
    iris.iris_token_logprobs_backward(z, rows, vocab, iris.LOGIT_DTYPES[dtype], t, t.shape[1], stats, g, dz, entropy=entropy if gh is not None else None,
                                      grad_entropy=gh, scale=scale, row_stride=z.stride(0) if rows > 1 else 0, grad_stride=dz.stride(0) if rows > 1 else 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,vocab,pad,offset,gpad,goffset,nt,with_h,scale", [
    (1, 1, 0, 0, 0, 0, 1, True, 1.0), (3, 7, 0, 0, 0, 0, 2, True, 0.5), (2, 33, 1, 1, 1, 1, 1, False, 1.0), (4, 1000, 0, 0, 0, 0, 1, True, 1.4),
    (3, 1001, 0, 0, 3, 2, 4, True, 1.0), (2, 4099, 5, 3, 0, 0, 128, False, 1.0), (2, 20000, 0, 0, 0, 0, 1, True, 1.0), (2, 50021, 0, 1, 0, 1, 3, True, 1.0),
    (1, 140001, 0, 0, 0, 0, 1, True, 1.0), (260, 515, 0, 0, 0, 0, 1, True, 1.0),
])
def test_score_gradient(dtype, rows, vocab, pad, offset, gpad, goffset, nt, with_h, scale):
    rng = np.random.default_rng(vocab + rows)
    values = logits_like(rng, rows, vocab)
    if vocab > 100:
        values[0, rng.random(vocab) < 0.3] = -np.inf
    _, z = strided(values, dtype, pad, offset)
    gstore, dz = strided(np.full((rows, vocab), SENTINEL), dtype, gpad, goffset)
    t = rng.integers(0, vocab, (rows, nt))
    t[:, -1] = t[:, 0]                       # a target that comes twice
    t[0, 0] = -1
    g, gh = rng.normal(0, 1, (rows, nt)).astype(np.float32), rng.random(rows).astype(np.float32) if with_h else None
    run_score_grad(z, dtype, torch.from_numpy(t).cuda(), torch.from_numpy(g).cuda(), torch.from_numpy(gh).cuda() if with_h else None, scale, dz)
    v, got = as64(z), as64(dz)
    for r in range(rows):
        want, size = ref.score_grad(v[r], scale, t[r], g[r].astype(np.float64), float(gh[r]) if with_h else 0.0)
        close(got[r], want, HALF_UNIT[dtype] * np.abs(want) + 3e-5 * size + SMALLEST[dtype], "dz")
    outside_untouched(gstore, dz, goffset)


@pytest.mark.parametrize("kind", ["most", "all", "one", "all_lowest", "lowest_and_one", "inf", "nan"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_score_gradient_masks_in_place(dtype, kind):
    rng = np.random.default_rng(2)
    _, z = strided(masked(rng, kind, 3, 2500, dtype), dtype, 0, 1)
    v = as64(z)
    t = torch.from_numpy(rng.integers(0, 2500, (3, 2))).cuda()
    g, gh = torch.randn(3, 2, device="cuda"), torch.rand(3, device="cuda")
    run_score_grad(z, dtype, t, g, gh, 1.0, z)
    got = as64(z)
    for r in range(3):
        if np.any(np.isnan(v[r])) or np.any(np.isposinf(v[r])):
            assert np.all(np.isnan(got[r]))
            continue
        want, size = ref.score_grad(v[r], 1.0, t[r].cpu().numpy(), as64(g[r]), gh[r].item())
        close(got[r], want, HALF_UNIT[dtype] * np.abs(want) + 3e-5 * size + SMALLEST[dtype], "dz")


def test_score_gradient_against_differences():
    """(f(z + h d) - f(z - h d)) / 2h of the forward call itself.  Error: h^2 / 6 of the third derivative (< 1e-3 at h = 0.05 for these
    directions of size 1) and the forward call's 3e-5 / h."""
    rng = np.random.default_rng(8)
    vocab, h = 400, 0.05
    z = torch.from_numpy(rng.normal(0, 1.5, (1, vocab)).astype(np.float32)).cuda()
    t = torch.tensor([[17, 301]], device="cuda")
    g, gh = torch.tensor([[0.7, -1.1]], device="cuda"), torch.tensor([0.9], device="cuda")
    dz = torch.empty_like(z)
    run_score_grad(z, "fp32", t, g, gh, 1.3, dz)

    def f(x):
        out = score(x, "fp32", t, 0, True, 1.3)
        return float((out["logprob"].double() * g).sum() + (out["entropy"].double() * gh).sum())

    for _ in range(8):
        d = torch.from_numpy(rng.normal(0, 1, (1, vocab)).astype(np.float32)).cuda()
        d[0, 17] += 3
        d /= d.norm()
        assert abs((f(z + h * d) - f(z - h * d)) / (2 * h) - float((dz.double() * d).sum())) < 1e-3 + 2e-3


# ------------------------------------------------------------------------------------------------ distillation
def teacher_of(rng, z, k, tail, noise=1.0):
    """A list from a noisy copy of the row."""
    y = np.where(np.isfinite(z), z, -50.0) + rng.normal(0, noise, z.shape)
    ids = np.argsort(-y, axis=1, kind="stable")[:, :k].astype(np.int64)
    v = np.take_along_axis(y, ids, 1)
    if tail:
        v = v - np.log(np.exp(y - y.max(1, keepdims=True)).sum(1, keepdims=True)) - y.max(1, keepdims=True)
    return ids, v.astype(np.float32)


def run_distill(z, dtype, ids, v, tail, scale=1.0, tscale=1.0, weight=None, dz=None, stats=True):
    rows, vocab = z.shape
    loss = torch.full((rows,), SENTINEL, device="cuda")
    st = torch.full((rows, 3), SENTINEL, device="cuda") if stats else None
    iris.iris_distill_topk(z, rows, vocab, iris.LOGIT_DTYPES[dtype], v, ids, ids.shape[1], loss, mode=int(tail), stats=st, weight=weight, dlogits=dz,
                           scale=scale, teacher_scale=tscale, row_stride=z.stride(0) if rows > 1 else 0,
                           grad_stride=dz.stride(0) if dz is not None and rows > 1 else 0)
    return loss, st


def check_distill(v, dtype, ids, tv, tail, scale, tscale, weight, loss, stats, dz):
    for r in range(v.shape[0]):
        want, dwant, size, dsize, lr = ref.distill(v[r], scale, ids[r], tv[r], tscale, tail)
        if loss is not None:
            close(loss[r].item(), want, 1e-5 + 1e-5 * size, "loss")
        if stats is not None:
            m, ls, _ = ref.log_softmax(v[r], scale)
            close(as64(stats[r]), [m, ls, lr], [0.0, 1e-5, 1e-5 + 1e-6 * abs(lr) if np.isfinite(lr) else 0.0], "stats")
        if dz is not None:
            w = 1.0 if weight is None else float(weight[r])
            close(dz[r], w * dwant, HALF_UNIT[dtype] * np.abs(w * dwant) + 3e-5 * abs(w) * dsize + SMALLEST[dtype], "dz")


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,vocab,pad,offset,gpad,goffset,k,scale,tscale", [
    (1, 1, 0, 0, 0, 0, 1, 1.0, 1.0), (2, 5, 0, 0, 0, 0, 5, 1.0, 1.0), (3, 9, 1, 1, 1, 1, 3, 0.5, 0.5), (4, 1000, 0, 0, 0, 0, 16, 0.5, 1.0),
    (3, 1001, 0, 0, 2, 3, 100, 1.0, 1.0), (2, 4099, 3, 5, 3, 5, 128, 1.0, 1.0), (2, 28672, 0, 0, 0, 0, 64, 0.5, 0.5), (3, 50021, 0, 1, 0, 1, 30, 1.0, 1.0),
    (2, 60001, 7, 0, 0, 0, 20, 1.0, 1.0), (1, 128000, 0, 0, 0, 0, 64, 1.0, 1.0), (2, 210007, 0, 3, 0, 3, 64, 1.0, 1.0), (200, 520, 0, 0, 0, 0, 8, 1.0, 1.0),
])
def test_distill(tail, dtype, rows, vocab, pad, offset, gpad, goffset, k, scale, tscale):
    rng = np.random.default_rng(vocab + k)
    store, z = strided(logits_like(rng, rows, vocab), dtype, pad, offset)
    v = as64(z)
    ids, tv = teacher_of(rng, v, k, tail)
    if k > 3:
        ids[0, -1], ids[-1, 1] = -1, vocab
    weight = (rng.random(rows) + 0.5).astype(np.float32)
    if rows > 2:
        weight[1] = 0
    gstore, dz = strided(np.full((rows, vocab), SENTINEL), dtype, gpad, goffset)
    d = [torch.from_numpy(x).cuda() for x in (ids, tv, weight)]
    loss, stats = run_distill(z, dtype, d[0], d[1], tail, scale, tscale, d[2], dz)
    check_distill(v, dtype, ids, tv, tail, scale, tscale, weight, loss, stats, as64(dz))
    outside_untouched(gstore, dz, goffset)
    outside_untouched(store, z, offset)
    # the loss alone, and the gradient from what it saved
    alone, saved = run_distill(z, dtype, d[0], d[1], tail, scale, tscale)
    check_distill(v, dtype, ids, tv, tail, scale, tscale, None, alone, saved, None)
    dz.fill_(SENTINEL)
    iris.iris_distill_topk_backward(z, rows, vocab, iris.LOGIT_DTYPES[dtype], d[1], d[0], k, saved, d[2], dz, mode=int(tail), scale=scale,
                                    teacher_scale=tscale, row_stride=z.stride(0) if rows > 1 else 0, grad_stride=dz.stride(0) if rows > 1 else 0)
    check_distill(v, dtype, ids, tv, tail, scale, tscale, weight, None, None, as64(dz))
    outside_untouched(gstore, dz, goffset)
    # in place
    run_distill(z, dtype, d[0], d[1], tail, scale, tscale, d[2], z)
    check_distill(v, dtype, ids, tv, tail, scale, tscale, weight, None, None, as64(z))
    outside_untouched(store, z, offset)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("kind", MASKS)
def test_distill_masks(tail, dtype, kind):
    rng = np.random.default_rng(9)
    vocab = 3001
    _, z = strided(masked(rng, kind, 3, vocab, dtype), dtype, 0, 3)
    v = as64(z)
    ids, tv = teacher_of(rng, rng.normal(0, 2, (3, vocab)), 12, tail)   # a teacher that does not know the mask
    dz = torch.empty_like(z)
    loss, stats = run_distill(z, dtype, torch.from_numpy(ids).cuda(), torch.from_numpy(tv).cuda(), tail, dz=dz)
    got = as64(dz)
    bad = np.array([np.any(np.isnan(x)) or np.any(np.isposinf(x)) for x in v])
    assert np.all(np.isnan(got[bad])) and bool(torch.isnan(loss[torch.from_numpy(bad).cuda()]).all())
    check_distill(v[~bad], dtype, ids[~bad], tv[~bad], tail, 1.0, 1.0, None, loss.cpu()[~bad], stats.cpu()[~bad], got[~bad])


@pytest.mark.parametrize("tail", [False, True])
def test_distill_lists(tail):
    """Empty lists, entries of no probability, a list of the whole vocabulary, one that holds all of the student's mass, a token listed twice."""
    rng = np.random.default_rng(10)
    vocab, k = 40, 40
    values = rng.normal(0, 1, (7, vocab))
    values[3] = -np.inf
    values[3, :4] = [1, 2, 3, 4]
    values[6] = -200.0
    values[6, 5] = 0.0
    _, z = strided(values, "fp32")
    v = as64(z)
    ids = np.stack([rng.permutation(vocab) for _ in range(7)]).astype(np.int64)
    tv = ref.log_softmax(rng.normal(0, 1, vocab), 1.0)[2].astype(np.float32) * np.ones((7, 1), np.float32)
    ids[0] = -1                                # nothing listed
    tv[1] = -np.inf                            # listed, nothing asked
    ids[2, 1:], tv[2, 0] = -1, 0.0             # one token, certain
    ids[3, 4:], ids[3, :4] = -1, [0, 1, 2, 3]  # all that the student has
    ids[4, 7] = ids[4, 6]
    if tail:
        tv[4] -= 0.7
    ids[5] = np.arange(vocab)                  # the whole vocabulary
    ids[6, 1:], ids[6, 0] = -1, 5              # the rest of the student's mass is below 1e-80
    dz = torch.empty_like(z)
    loss, stats = run_distill(z, "fp32", torch.from_numpy(ids).cuda(), torch.from_numpy(tv).cuda(), tail, dz=dz)
    check_distill(v, "fp32", ids, tv, tail, 1.0, 1.0, None, loss, stats, as64(dz))
    got = dz.clone()
    iris.iris_distill_topk_backward(z, 7, vocab, iris.IRIS_F32, torch.from_numpy(tv).cuda(), torch.from_numpy(ids).cuda(), k, stats,
                                    torch.ones(7, device="cuda"), dz, mode=int(tail))
    check_distill(v, "fp32", ids, tv, tail, 1.0, 1.0, None, None, None, as64(dz))
    assert float((got - dz).abs().max()) < 1e-5
    none = torch.empty(7, 0, device="cuda")
    loss, _ = run_distill(z, "fp32", none.long(), none, tail, dz=dz)
    assert float(loss.abs().max()) < 2e-5 and float(dz.abs().max()) < 1e-5


def test_weight_zero_gives_zero_whatever_the_row_holds():
    z = torch.full((3, 600), math.nan, device="cuda")
    z[1] = 0.5
    ids, tv = torch.zeros(3, 1, dtype=torch.int64, device="cuda"), torch.zeros(3, 1, device="cuda")
    w = torch.tensor([0.0, 0.0, 1.0], device="cuda")
    dz = torch.empty_like(z)
    _, st = run_distill(z, "fp32", ids, tv, False, weight=w, dz=dz)
    assert bool((dz[:2] == 0).all()) and bool(torch.isnan(dz[2]).all())
    iris.iris_distill_topk_backward(z, 3, 600, iris.IRIS_F32, tv, ids, 1, st, w, dz)
    assert bool((dz[:2] == 0).all()) and bool(torch.isnan(dz[2]).all())


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_against_differences(tail):
    """As for the scores: h = 0.05, directions of size 1."""
    rng = np.random.default_rng(12)
    vocab, k, h = 300, 10, 0.05
    z = torch.from_numpy(rng.normal(0, 1.5, (1, vocab)).astype(np.float32)).cuda()
    ids, tv = [torch.from_numpy(x).cuda() for x in teacher_of(rng, as64(z), k, tail)]
    dz = torch.empty_like(z)
    run_distill(z, "fp32", ids, tv, tail, 1.2, 0.8, dz=dz)

    def f(x):
        return run_distill(x, "fp32", ids, tv, tail, 1.2, 0.8)[0].double().item()

    for _ in range(8):
        d = torch.from_numpy(rng.normal(0, 1, (1, vocab)).astype(np.float32)).cuda()
        d[0, ids[0, 0]] += 3
        d /= d.norm()
        assert abs((f(z + h * d) - f(z - h * d)) / (2 * h) - float((dz.double() * d).sum())) < 1e-3 + 2e-3


def test_gradient_into_other_columns_of_the_same_matrix():
    rng = np.random.default_rng(13)
    both = torch.from_numpy(rng.normal(0, 1, (5, 2000)).astype(np.float32)).cuda().bfloat16()
    z, dz = both[:, :1000], both[:, 1000:]
    v = as64(z)
    ids, tv = teacher_of(rng, v, 6, False)
    run_distill(z, "bf16", torch.from_numpy(ids).cuda(), torch.from_numpy(tv).cuda(), False, dz=dz)
    check_distill(v, "bf16", ids, tv, False, 1.0, 1.0, None, None, None, as64(dz))


# ------------------------------------------------------------------------------------------------ scales, and calls in a row
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("scale", [1e-6, 0.01, 30.0, 1e4, 1e9])
def test_scales_far_from_one(dtype, scale):
    """Exponents y = scale (z - max) log2(e) carry 3 roundings of 2^-24 each; what they weigh falls as 2^y: errors as in the other tests, except
    that log probabilities scale with y (1e-6 of the value)."""
    rng = np.random.default_rng(21)
    values = logits_like(rng, 3, 3001)
    values[1, rng.random(3001) < 0.5] = -np.inf
    _, z = strided(values, dtype, 0, 1)
    t = torch.from_numpy(rng.integers(0, 3001, (3, 2))).cuda()
    out = score(z, dtype, t, 9, True, scale)
    check_score(z, out, t, 9, scale)
    v = as64(z)
    g, gh = torch.ones(3, 2, device="cuda") / scale, torch.ones(3, device="cuda") / scale
    dz = torch.empty_like(z)
    run_score_grad(z, dtype, t, g, gh, scale, dz, out["stats"], out["entropy"])
    for r in range(3):
        want, size = ref.score_grad(v[r], scale, t[r].cpu().numpy(), as64(g[r]), gh[r].item())
        close(as64(dz[r]), want, HALF_UNIT[dtype] * np.abs(want) + 3e-5 * size + SMALLEST[dtype], "dz")


def test_calls_in_a_row_wait_for_one_another():
    """Kernels may begin while the one before them ends; each has to see all that was written before it in the stream."""
    rng = np.random.default_rng(22)
    vocab, rows = 20000, 40
    zs = [torch.from_numpy(logits_like(rng, rows, vocab)).cuda().bfloat16() for _ in range(2)]
    t = torch.from_numpy(rng.integers(0, vocab, (rows, 1))).cuda()
    g = torch.ones(rows, 1, device="cuda")
    ids = [z.float().topk(16, dim=1).indices for z in zs]
    tv = torch.zeros(rows, 16, device="cuda")
    st, lp, loss, st3 = (torch.empty(rows, n, device="cuda") for n in (2, 1, 1, 3))
    ones = torch.ones(rows, device="cuda")

    def chain(z, i, buf, dz, sync):
        steps = [
            lambda: buf.copy_(z),
            lambda: iris.iris_token_logprobs(buf, rows, vocab, iris.IRIS_BF16, targets=t, n_targets=1, logprob=lp, stats=st),
            lambda: iris.iris_token_logprobs_backward(buf, rows, vocab, iris.IRIS_BF16, t, 1, st, g, buf),      # in place
            lambda: iris.iris_distill_topk(buf, rows, vocab, iris.IRIS_BF16, tv, i, 16, loss, stats=st3),       # of the gradient, as logits
            lambda: iris.iris_distill_topk_backward(buf, rows, vocab, iris.IRIS_BF16, tv, i, 16, st3, ones, dz),
            lambda: iris.iris_distill_topk(dz, rows, vocab, iris.IRIS_BF16, tv, i, 16, loss, dlogits=dz),       # in place
        ]
        for s in steps:
            s()
            if sync:
                torch.cuda.synchronize()
        return dz.clone(), loss.clone()

    buf, dz = torch.empty_like(zs[0]), torch.empty_like(zs[0])
    want = [chain(z, i, buf, dz, True) for z, i in zip(zs, ids)]
    got = [chain(zs[n % 2], ids[n % 2], buf, dz, False) for n in range(60)]
    torch.cuda.synchronize()
    for n, (a, b) in enumerate(got):
        assert torch.equal(a, want[n % 2][0]) and torch.equal(b, want[n % 2][1]), n


def test_calls_in_a_cuda_graph():
    rng = np.random.default_rng(23)
    _, z = strided(logits_like(rng, 8, 40000), "bf16")
    want = score(z, "bf16", None, 20)
    out = {k: torch.zeros_like(v) for k, v in want.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            iris.iris_token_logprobs(z, 8, 40000, iris.IRIS_BF16, top_k=20, entropy=out["entropy"], stats=out["stats"], top_ids=out["top_ids"],
                                     top_logprob=out["top_logprob"])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out["top_ids"], want["top_ids"]) and torch.equal(out["stats"], want["stats"]) and torch.equal(out["entropy"], want["entropy"])


# ------------------------------------------------------------------------------------------------ many rows, and rows beyond shared memory
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab,top,pad", [(9000, 128, 0), (20001, 5, 0), (36864, 64, 3), (70000, 128, 0)])
@pytest.mark.parametrize("kind", ["random", "masked", "few_left", "four_threads", "constant", "rising"])
def test_alternatives_of_many_rows(dtype, vocab, top, pad, kind):
    """As many rows as keep a block for each: against a stable sort of all rows, and the definition for three."""
    rows = 380
    gen = torch.Generator(device="cuda").manual_seed(vocab + top)
    x = torch.randn(rows, vocab, device="cuda", generator=gen) * 3
    j = torch.arange(vocab, device="cuda")
    if kind == "masked":
        x[torch.rand(x.shape, device="cuda", generator=gen) < 0.99] = -math.inf
    elif kind == "few_left":
        x[:, torch.rand(vocab, device="cuda", generator=gen) > 3 / vocab] = -math.inf
    elif kind == "four_threads":                       # what a block's threads 3 .. 6 read holds all that is large
        x = torch.where((j // (16 // TORCH[dtype].itemsize) % 256 - 3).clamp(0, 3) == j // (16 // TORCH[dtype].itemsize) % 256 - 3, 20.0, 0.0) + x * 1e-2
    elif kind == "constant":
        x[:] = 0.5
    elif kind == "rising":
        x = (j * 1e-3).expand(rows, vocab)
    store = torch.zeros(rows, vocab + pad, dtype=TORCH[dtype], device="cuda")
    z = store[:, :vocab]
    z.copy_(x)
    out = score(z, dtype, None, top)
    want = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(out["top_ids"], want)
    few = torch.tensor([0, rows // 2, rows - 1], device="cuda")
    check_score(z[few], {k: v[few] for k, v in out.items()}, None, top, 1.0)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype,vocab,offset", [("fp32", 400003, 1), ("bf16", 900001, 0), ("bf16", 800000, 0)])
def test_distill_rows_beyond_shared_memory(tail, dtype, vocab, offset):
    rng = np.random.default_rng(31)
    store, z = strided(logits_like(rng, 2, vocab), dtype, 0, offset)
    v = as64(z)
    ids, tv = teacher_of(rng, v, 50, tail)
    ids[1, 3] = ids[1, 4]
    d = [torch.from_numpy(a).cuda() for a in (ids, tv)]
    w = np.array([1.0, 0.25], np.float32)
    dz = torch.empty_like(z)
    for target in (dz, z):                             # apart, then in place
        loss, stats = run_distill(z, dtype, d[0], d[1], tail, weight=torch.from_numpy(w).cuda(), dz=target)
        check_distill(v, dtype, ids, tv, tail, 1.0, 1.0, w, loss, stats, as64(target))
    outside_untouched(store, z, offset)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_many_rows_of_unlike_places(tail):
    """Enough rows that each block takes several, every row at another place in its 16 bytes, the gradient's rows elsewhere."""
    rng = np.random.default_rng(32)
    rows, vocab, k = 1500, 5003, 12
    values = logits_like(rng, rows, vocab)
    for gpad in (2, 3):                                # as the logits' rows, and not
        store, z = strided(values, "fp16", 2, 1)
        v = as64(z)
        ids, tv = teacher_of(rng, v, k, tail)
        ids[::3, -1] = -1
        ids[7, 0] = ids[7, 1]
        gstore, dz = strided(np.full((rows, vocab), SENTINEL), "fp16", gpad, 1)
        w = (rng.random(rows) * 64).astype(np.float32)
        w[::5] = 0
        d = [torch.from_numpy(a).cuda() for a in (ids, tv, w)]
        loss, stats = run_distill(z, "fp16", d[0], d[1], tail, weight=d[2], dz=dz)
        check_distill(v, "fp16", ids, tv, tail, 1.0, 1.0, w, loss, stats, as64(dz))
        outside_untouched(gstore, dz, 1)
        if gpad == 2:
            run_distill(z, "fp16", d[0], d[1], tail, weight=d[2], dz=z)
            check_distill(v, "fp16", ids, tv, tail, 1.0, 1.0, w, None, None, as64(z))
            outside_untouched(store, z, 1)
