"""Operators on logits where they went wrong once: finite masks off the teacher's list, long rows, tokens listed twice, scales near
the type's largest, rows of NaN, 32-bit gradients, graphs.

Tolerances are those of test_gpu_logit_ops.py unless a test derives its own.
"""
import math
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

import logit_ref as ref
import paper_2511_12500_b200 as iris
from paper_2511_12500_b200 import binding
from test_gpu_logit_ops import HALF_UNIT, SMALLEST, TORCH, as64, check_score, close, logits_like, run_distill, run_score_grad, score, strided

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ finite masks off the teacher's list
def masked_off_list(z, scale, ids, tv):
    """Loss, gradient, ln of the sum off the list and the sizes of the first two's terms, in 64 bits, with the tokens off the list counted from
    their own largest (64 bits do not hold ln n beside 1e38).  A remainder below 1e-5 is dropped where the probability off the list is below
    2^-126."""
    m, ls, lq = ref.log_softmax(z, scale)
    there = ids >= 0
    p = np.where(there, np.exp(tv.astype(np.float64)), 0.0)
    rest = max(0.0, 1.0 - p.sum())
    off = np.ones(z.size, dtype=bool)
    off[ids[there]] = False
    top = z[off].max()
    y = np.exp(scale * (z - top), where=off, out=np.zeros(z.size))
    down, lo = scale * (m - top), np.log(y.sum())                      # ln of the sum off the list = lo - down
    if rest < 1e-5 and lo - down - ls < -126 * math.log(2):
        rest = 0.0
    q = np.exp(lq)
    dz, dsize = (p.sum() + rest) * q - rest * y / y.sum(), (p.sum() + rest) * q + rest * y / y.sum()
    dz[ids[there]] -= p[there]
    dsize[ids[there]] += p[there]
    terms = np.array([x * (np.log(x) - lq[j]) for j, x in zip(ids, p) if j >= 0 and x > 0] + ([rest * np.log(rest), rest * ls, -rest * lo, rest * down] if rest else []))
    return terms.sum(), scale * dz, lo - down, np.abs(terms).sum(), scale * dsize


MASK_VALUES = [(d, m) for d in ("bf16", "fp16", "fp32") for m in (None, -1e9, -1e4) if (d, m) != ("fp16", -1e9)]   # None: the type's lowest


def rows_with_masked_rest(dtype, mask, rows, vocab, k, p_rest, offset, others):
    """Rows in which all tokens off the list are masked, by one value or by three."""
    rng = np.random.default_rng(vocab)
    low = float(torch.finfo(TORCH[dtype]).min) if mask is None else mask
    values = np.full((rows, vocab), low)
    if others:
        values[:, ::3] = low / 2
        values[:, 1::7] = -np.inf
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int64)
    np.put_along_axis(values, ids, rng.normal(0, 2, (rows, k)), 1)
    p = rng.random((rows, k)) + 0.1
    tv = np.log(p / p.sum(1, keepdims=True) * (1 - p_rest)).astype(np.float32)
    absent = rng.permutation(k)[0]
    if p_rest > 1e-3:
        values[0, ids[0, absent]] = low                                # an absent entry's token is off the list too
        ids[0, absent] = -1
    store, z = strided(values, dtype, 0, offset)
    return store, z, ids, tv


def check_masked_rest(dtype, z, v, ids, tv, scale, weight, what, loss=None, stats=None, dz=None):
    for r in range(v.shape[0]):
        want, dwant, lr, size, dsize = masked_off_list(v[r], scale, ids[r], tv[r])
        w = float(weight[r])
        if loss is not None:
            close(loss[r].item(), want, 1e-5 + 1e-5 * size, what + " loss")
        if stats is not None:
            lr = max(lr, -float(np.finfo(np.float32).max))
            close(as64(stats[r]), [*ref.log_softmax(v[r], scale)[:2], lr], [0.0, 1e-5, 1e-5 + 1e-6 * abs(lr)], what + " stats")
        if dz is not None:
            close(dz[r], w * dwant, HALF_UNIT[dtype] * np.abs(w * dwant) + 3e-5 * abs(w) * dsize + SMALLEST[dtype], what + " dz")


def run_masked_rest(dtype, mask, scale, p_rest, rows, vocab, offset, others, gradients, losses):
    k = 12
    store, z, ids, tv = rows_with_masked_rest(dtype, mask, rows, vocab, k, p_rest, offset, others)
    v = as64(z)
    weight = np.linspace(0.5, 64 if dtype == "fp16" else 1.5, rows).astype(np.float32)
    i, t, w = [torch.from_numpy(x).cuda() for x in (ids, tv, weight)]
    dz = torch.empty_like(z)
    loss, stats = run_distill(z, dtype, i, t, True, scale, weight=w, dz=dz)
    alone, saved = run_distill(z, dtype, i, t, True, scale)
    if losses:
        check_masked_rest(dtype, z, v, ids, tv, scale, weight, "fused", loss=loss, stats=stats)
        check_masked_rest(dtype, z, v, ids, tv, scale, weight, "alone", loss=alone, stats=saved)
    if gradients:
        check_masked_rest(dtype, z, v, ids, tv, scale, weight, "fused", dz=as64(dz))
        where = (z, rows, vocab, iris.LOGIT_DTYPES[dtype], t, i, k, saved, w)
        strides = dict(row_stride=z.stride(0), grad_stride=z.stride(0)) if rows > 1 else {}
        iris.iris_distill_topk_backward(*where, dz, mode=iris.IRIS_DISTILL_TAIL, scale=scale, **strides)
        check_masked_rest(dtype, z, v, ids, tv, scale, weight, "backward", dz=as64(dz))
        keep = z.clone()
        iris.iris_distill_topk_backward(*where, z, mode=iris.IRIS_DISTILL_TAIL, scale=scale, **strides)
        check_masked_rest(dtype, z, v, ids, tv, scale, weight, "backward in place", dz=as64(z))
        z.copy_(keep)
        run_distill(z, dtype, i, t, True, scale, weight=w, dz=z)
        check_masked_rest(dtype, z, v, ids, tv, scale, weight, "fused in place", dz=as64(z))


@pytest.mark.parametrize("dtype,mask", MASK_VALUES)
@pytest.mark.parametrize("scale", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("p_rest", [0.1, 0.6])
@pytest.mark.parametrize("rows,vocab,offset,others", [(4, 3001, 3, False), (3, 20000, 0, True), (1, 128000, 0, False), (2, 60001, 1, True)])
def test_remainder_over_finite_masks(dtype, mask, scale, p_rest, rows, vocab, offset, others):
    """A student whose tokens off the list are all masked by a finite value: the remainder's gradient is spread over them by their own softmax."""
    run_masked_rest(dtype, mask, scale, p_rest, rows, vocab, offset, others, True, False)


@pytest.mark.parametrize("dtype,vocab", [("fp32", 400003), ("bf16", 900001)])
@pytest.mark.parametrize("mask", [None, -1e9])
def test_remainder_over_finite_masks_beyond_shared_memory(dtype, vocab, mask):
    run_masked_rest(dtype, mask, 1.0, 0.1, 2, vocab, 1, True, True, False)


# ------------------------------------------------------------------------------------------------ what rounding leaves of no remainder
@pytest.mark.parametrize("dtype,mask", MASK_VALUES)
@pytest.mark.parametrize("scale", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("p_rest", [0.0, 6e-8, 0.1])
@pytest.mark.parametrize("rows,vocab", [(4, 3001), (1, 128000)])
def test_no_remainder_over_finite_masks(dtype, mask, scale, p_rest, rows, vocab):
    """A list that holds all of the teacher's mass: what rounding leaves of 1 - sum p must not meet ln q_r of -1e9."""
    run_masked_rest(dtype, mask, scale, p_rest, rows, vocab, 0, False, True, True)


# ------------------------------------------------------------------------------------------------ long rows
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_sums_of_long_rows(dtype):
    """2^24 columns of which seven in eight are 0.7 times as probable as the eighth: a chain of all of a thread's terms (4096 in a lane) rounds
    each to the same side and is 3e-5 off; the tolerance is that of short rows."""
    vocab, rows = 1 << 24, 1
    z = torch.full((rows, vocab), math.log(0.7), dtype=TORCH[dtype], device="cuda")
    z[:, ::8] = 0.0
    x = z.double()
    ls = float(torch.logsumexp(x, 1)[0])
    lq = x[0] - ls
    h = float(-(lq.exp() * lq).sum())
    t = torch.tensor([[0, 1]], device="cuda")
    for entropy in (True, False):
        for top in (0, 5):
            out = score(z, dtype, t, top, entropy)
            close(as64(out["stats"][0]), [0.0, ls], [0.0, 1e-5], "stats")
            close(as64(out["logprob"][0]), as64(lq[:2]), 1e-5 + 1e-6 * ls, "logprob")
            if entropy:
                close(out["entropy"][0].item(), h, 3e-5 + 1e-6 * h, "entropy")
    ids = torch.arange(16, device="cuda")[None]
    tv = torch.log_softmax(torch.arange(16, device="cuda") * -0.1, 0)[None].float().contiguous()
    for tail in (False, True):
        for dz in (None, torch.empty_like(z)):
            loss, st = run_distill(z, dtype, ids, tv, tail, dz=dz)
            close(as64(st[0, :2]), [0.0, ls], [0.0, 1e-5], "stats")
            want = float((tv.double().exp() * (tv.double() - lq[:16])).sum())
            close(loss[0].item(), want, 1e-5 + 1e-5 * 20, "loss")


# ------------------------------------------------------------------------------------------------ tokens listed twice
@pytest.mark.parametrize("rows,vocab", [(600, 5000), (40, 60000)])
@pytest.mark.parametrize("grad", [True, False])
def test_tokens_listed_twice_give_the_same_bits(rows, vocab, grad):
    """Every token is listed by two warps: which of them is counted must not depend on which comes first."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    z = torch.randn(rows, vocab, device="cuda", generator=gen) * 2
    half = torch.rand(rows, vocab, device="cuda", generator=gen).topk(64, dim=1).indices
    ids = torch.cat([half, half.flip(1)], 1).contiguous()
    tv = torch.log_softmax(torch.randn(rows, 128, device="cuda", generator=gen), 1).sub(0.3).contiguous()
    dz = torch.empty_like(z) if grad else None
    loss, stats = run_distill(z, "fp32", ids, tv, True, dz=dz)
    first = [x.clone() for x in (loss, stats, dz) if x is not None]
    for _ in range(60):
        loss, stats = run_distill(z, "fp32", ids, tv, True, dz=dz)
        for a, b in zip(first, [x for x in (loss, stats, dz) if x is not None]):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ scales near the type's largest
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [1e30, 1e36, 2e38])
def test_scales_near_the_largest(dtype, scale):
    """Differences of half a unit become 1e30 and more: one token, or equal ones, have all the probability, and
    scale g_H ln 2 times a cut exponent overflows.  (scale log2(e) itself does from 2.4e38 on: refused.)"""
    values = np.full((3, 900), -1.0)
    values[0, 400], values[1, [5, 6, 700]], values[2, ::2] = -0.5, -0.5, -np.inf
    values[2, 31] = -0.75
    _, z = strided(values, dtype)
    t = torch.tensor([[400, 3], [6, 7], [31, 0]], device="cuda")
    out = score(z, dtype, t, 5, True, scale)
    check_score(z, out, t, 5, scale)
    g, gh = torch.full((3, 2), 1 / scale, device="cuda"), torch.ones(3, device="cuda")
    dz = torch.empty_like(z)
    run_score_grad(z, dtype, t, g, gh, scale, dz, out["stats"], out["entropy"])
    g64, v = as64(g), as64(z)
    for r in (0, 2):                                       # row 1 has entropy, whose gradient is rounding times the scale
        want, _ = ref.score_grad(v[r], scale, t[r].cpu().numpy(), g64[r], 1.0)
        close(as64(dz[r]), want, HALF_UNIT[dtype] * np.abs(want) + 3e-5, "dz")
    ids, tv = t.clone(), torch.zeros(3, 2, device="cuda")
    loss, st = run_distill(z, dtype, ids[:, :1].contiguous(), tv[:, :1].contiguous(), False, scale, dz=dz, weight=torch.full((3,), 1 / scale, device="cuda"))
    close(as64(loss), [0.0, math.log(3), 0.0], 1e-5, "loss")
    close(as64(dz[1, [5, 6, 700]]), [1 / 3, -2 / 3, 1 / 3], 2.0 ** -8 if dtype == "bf16" else 3e-5, "dz")


@pytest.mark.parametrize("tscale", [2.0, 1e30, 3e38])
def test_teacher_values_times_teacher_scale_beyond_the_type(tscale):
    """p = softmax(teacher_scale v): only differences of the values count, also where the products would overflow."""
    low = float(np.finfo(np.float32).min)
    v = np.array([[2.0, 1.0, 2.0, -3.0], [low, low, low, low], [low, 3.0, low, -np.inf], [3e38, 3e38, -3e38, 0.0]], np.float32)
    want = np.array([[0.5, 0, 0.5, 0], [0.25] * 4, [0, 1, 0, 0], [0.5, 0.5, 0, 0]])
    if tscale == 2.0:
        e = np.exp(2.0 * (v[0].astype(np.float64) - 2))
        want[0] = e / e.sum()
    rng = np.random.default_rng(1)
    _, z = strided(rng.normal(0, 1, (4, 300)), "fp32")
    x = as64(z)
    ids = torch.arange(4, device="cuda").repeat(4, 1).contiguous()
    dz = torch.empty_like(z)
    loss, st = run_distill(z, "fp32", ids, torch.from_numpy(v).cuda(), False, 1.0, tscale, dz=dz)
    back = torch.empty_like(z)
    iris.iris_distill_topk_backward(z, 4, 300, iris.IRIS_F32, torch.from_numpy(v).cuda(), ids, 4, st, torch.ones(4, device="cuda"), back, teacher_scale=tscale)
    for r in range(4):
        lq = ref.log_softmax(x[r], 1.0)[2]
        p = want[r]
        close(loss[r].item(), sum(a * (math.log(a) - b) for a, b in zip(p, lq) if a > 0), 1e-4, "loss")
        dwant = np.exp(lq)
        dwant[:4] -= p
        close(as64(dz[r]), dwant, 1e-4 * np.abs(dwant) + 3e-5, "dz")
        close(as64(back[r]), dwant, 1e-4 * np.abs(dwant) + 3e-5, "backward")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tail", [False, True])
def test_listed_tokens_masked_by_the_lowest_value(dtype, tail):
    """p times a log probability of -4.8e38 is in range where p is 0.1."""
    scale, low = 1 / 0.7, float(torch.finfo(TORCH[dtype]).min)
    rng = np.random.default_rng(60)
    values = rng.normal(0, 1, (2, 400))
    values[:, [7, 9]] = low
    _, z = strided(values, dtype)
    v = as64(z)
    ids = np.array([[1, 2, 7, 9]] * 2)
    p = np.array([0.5, 0.3, 0.1, 0.05])
    tv = np.log(p).astype(np.float32)[None].repeat(2, 0)
    dz = torch.empty_like(z)
    loss, st = run_distill(z, dtype, torch.from_numpy(ids).cuda(), torch.from_numpy(tv).cuda(), tail, scale, 1.0, dz=dz)
    for r in range(2):
        want, dwant, size, dsize, _ = ref.distill(v[r], scale, ids[r], tv[r], 1.0, tail)
        assert 1e37 < want < 3e38
        close(loss[r].item(), want, 1e-5 * size, "loss")
        close(as64(dz[r]), dwant, HALF_UNIT[dtype] * np.abs(dwant) + 3e-5 * dsize + SMALLEST[dtype], "dz")


# ------------------------------------------------------------------------------------------------ rows of NaN
@pytest.mark.parametrize("grad", [True, False])
def test_a_row_of_nan_gives_a_loss_of_nan_whatever_is_asked(grad):
    z = torch.zeros(4, 700, device="cuda")
    z[0, 600], z[1, 600], z[2, 600] = math.nan, math.inf, math.nan
    ids = torch.tensor([[-1, -1], [3, 5], [3, 600], [-1, -1]], device="cuda")
    tv = torch.zeros(4, 2, device="cuda")
    tv[1] = -math.inf                                      # listed, nothing asked
    dz = torch.empty_like(z) if grad else None
    loss, _ = run_distill(z, "fp32", ids, tv, False, dz=dz)
    assert torch.isnan(loss).tolist() == [True, True, True, False] and loss[3].item() == 0
    if grad:
        assert bool(torch.isnan(dz[:3]).all()) and bool((dz[3] == 0).all())


# ------------------------------------------------------------------------------------------------ 32-bit gradients
def test_32_bit_gradients_to_a_few_roundings():
    """Root mean square of relative errors where q > 2^-8, statistics given to half a unit.  The exponent y (|y| < 8, raised by 8: a result below 8)
    carries the roundings of z - m (< 8), y and the offset (< 4), half units 2^-22, 2^-22 and 2^-23 of 2^y's ln 2, root mean squares 1 / sqrt 3 of that;
    2^y and three products 2^-22 and 2^-24 likewise: 2e-7 together in the mean.  Exponents near 32 would carry 2^-20: 5e-7."""
    rng = np.random.default_rng(40)
    rows, vocab = 60, 2000
    values = rng.normal(0, 2.5, (rows, vocab))
    for r in range(rows):
        values[r, rng.integers(0, vocab, 40)] += 6
    _, z = strided(values, "fp32")
    v = as64(z)
    stats, lqs = zip(*[((m, ls), lq) for m, ls, lq in (ref.log_softmax(x, 1.0) for x in v)])
    st = torch.tensor(stats, dtype=torch.float32, device="cuda")
    t = torch.zeros(rows, 1, dtype=torch.int64, device="cuda")
    dz = torch.empty_like(z)
    iris.iris_token_logprobs_backward(z, rows, vocab, iris.IRIS_F32, t, 1, st, torch.full((rows, 1), -1.0, device="cuda"), dz)
    st3 = torch.cat([st, torch.zeros(rows, 1, device="cuda")], 1).contiguous()
    kd = torch.empty_like(z)
    iris.iris_distill_topk_backward(z, rows, vocab, iris.IRIS_F32, torch.zeros(rows, 1, device="cuda"), t, 1, st3, torch.ones(rows, device="cuda"), kd)
    q = np.exp(np.stack(lqs))
    sel = q > 2.0 ** -8
    sel[:, 0] = False
    assert sel.sum() > 500
    for got in (as64(dz), as64(kd)):
        assert np.sqrt(np.mean((got[sel] / q[sel] - 1) ** 2)) < 3e-7


# ------------------------------------------------------------------------------------------------ graphs and threads
@pytest.mark.parametrize("dtype,vocab", [("bf16", 3000), ("fp16", 40000), ("fp32", 400003)])
@pytest.mark.parametrize("tail", [False, True])
def test_distillation_in_a_cuda_graph(dtype, vocab, tail):
    rng = np.random.default_rng(41)
    rows, k = 5, 16
    _, z = strided(logits_like(rng, rows, vocab), dtype)
    ids = z.float().topk(k, dim=1).indices.contiguous()
    tv = torch.log_softmax(torch.randn(rows, k, device="cuda"), 1).sub(0.1).contiguous()
    w = torch.rand(rows, device="cuda")
    loss, st, alone = torch.zeros(rows, device="cuda"), torch.zeros(rows, 3, device="cuda"), torch.zeros(rows, device="cuda")
    dz, back = torch.zeros_like(z), torch.zeros_like(z)

    def calls():
        where = (z, rows, vocab, iris.LOGIT_DTYPES[dtype], tv, ids, k)
        iris.iris_distill_topk(*where, loss, mode=int(tail), stats=st, weight=w, dlogits=dz)
        iris.iris_distill_topk(*where, alone, mode=int(tail))
        iris.iris_distill_topk_backward(*where, st, w, back, mode=int(tail))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                          # the first calls of these sizes: their queries run while the stream is captured
        calls()
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in (loss, st, alone, dz, back)]
    for x in (loss, st, alone, dz, back):
        x.zero_()
    calls()
    torch.cuda.synchronize()
    for a, b in zip(got, (loss, st, alone, dz, back)):
        assert torch.equal(a, b) and float(a.float().abs().max()) > 0


@pytest.mark.parametrize("vocab", [700, 9000, 41000])
def test_calls_from_several_threads(vocab):
    """Each thread with its own stream and outputs; the first of them sets up the kernels while the others call them."""
    rows, k, n = 6, 8, 8
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    zs = [torch.randn(rows, vocab, device="cuda", generator=gen).half() for _ in range(n)]
    ids = [z.float().topk(k, dim=1).indices.contiguous() for z in zs]
    tv = torch.log_softmax(torch.randn(rows, k, device="cuda", generator=gen), 1).sub(0.1).contiguous()
    losses, grads = torch.zeros(2, n, rows, device="cuda"), [[torch.zeros_like(z) for z in zs] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(n)]
    torch.cuda.synchronize()

    def call(turn, i):
        for _ in range(20):
            iris.iris_distill_topk(zs[i], rows, vocab, iris.IRIS_F16, tv, ids[i], k, losses[turn, i], mode=iris.IRIS_DISTILL_TAIL, dlogits=grads[turn][i],
                                   stream=streams[i])

    with ThreadPoolExecutor(n) as pool:
        list(pool.map(lambda i: call(0, i), range(n)))
    torch.cuda.synchronize()
    for i in range(n):
        call(1, i)
    torch.cuda.synchronize()
    assert torch.equal(losses[0], losses[1]) and all(torch.equal(a, b) for a, b in zip(*grads)) and float(losses.abs().min()) > 0


# ------------------------------------------------------------------------------------------------ tensors of a call
def test_tensors_that_are_right_pass_at_once_and_by_the_slower_look(monkeypatch):
    """Contiguous, strided, of more dimensions, longer than needed, parameters, addresses: the same answers from the extension and without it."""
    rng = np.random.default_rng(50)
    rows, vocab = 6, 500
    full = torch.from_numpy(rng.normal(0, 2, (rows + 1, vocab + 36)).astype(np.float32)).cuda().bfloat16()
    view = full[1:, 5:vocab + 5]
    t = torch.from_numpy(rng.integers(0, vocab, (rows + 2, 2))).cuda()
    some = view.contiguous()
    forms = [(view, vocab + 36), (some, 0), (some, vocab), (some.view(2, 3, vocab), 0), (some.view(-1), 0), (some.data_ptr(), 0),
             (torch.nn.Parameter(some, requires_grad=False), 0), (some.clone().requires_grad_(), 0), (full.view(-1)[vocab + 41:], vocab + 36)]
    look = binding._look
    slow = []
    monkeypatch.setattr(binding, "_look", lambda *a: slow.append(1) or look(*a))
    for accept in (binding._accept, binding._none):
        monkeypatch.setattr(binding, "_accept", accept)
        for z, stride in forms:
            want = score(view, "bf16", t[:rows], 7, stride=vocab + 36) if stride == vocab + 36 else score(some, "bf16", t[:rows], 7)
            slow.clear()
            out = {k: torch.zeros_like(v) for k, v in want.items()}
            iris.iris_token_logprobs(z, rows, vocab, iris.IRIS_BF16, targets=t, n_targets=2, top_k=7, row_stride=stride, **out)
            assert all(torch.equal(out[k], want[k]) for k in want)
            assert len(slow) == (accept is binding._none or type(z) is torch.nn.Parameter)      # a parameter is not of the type itself


def test_tensors_that_are_wrong_are_refused_on_the_gpu():
    rows, vocab = 4, 300
    z, t = torch.zeros(rows, vocab, device="cuda"), torch.zeros(rows, 1, dtype=torch.int64, device="cuda")
    st, g, dz = torch.zeros(rows, 2, device="cuda"), torch.ones(rows, 1, device="cuda"), torch.zeros(rows, vocab, device="cuda")
    one = torch.ones(1, device="cuda").expand(rows, 1)                                   # what autograd hands to the backward of a sum
    for change in (dict(targets=t.int()), dict(grad_logprob=one), dict(grad_logprob=g[:3]), dict(stats=st.double()), dict(stats=st[:, :1]),
                   dict(dlogits=dz.half()), dict(dlogits=torch.zeros(rows, vocab + 4, device="cuda")[:, :vocab]), dict(logits=z[:3]), dict(logits=z.cpu())):
        with pytest.raises(iris.IrisError) as e:
            iris.iris_token_logprobs_backward(**{**dict(logits=z, rows=rows, vocab=vocab, dtype=iris.IRIS_F32, targets=t, n_targets=1, stats=st, grad_logprob=g,
                                                        dlogits=dz), **change})
        assert e.value.code == iris.IRIS_ERR_ARG and next(iter(change)) in str(e.value)
