"""The operators around the head against their 64-bit definitions: embedding lookup and gradient, layer norm and gradient, verification of drafts."""
import math

import pytest
import torch

import paper_2511_12500_b200 as iris
import head_ref as ref

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
KIND = {BF16: iris.IRIS_BF16, FP16: iris.IRIS_F16, FP32: iris.IRIS_F32}
TYPES = [BF16, FP16, FP32]
GUARD = 7.0   # what lies outside rows and has to stay


def rows(n, dim, dtype, pad=0, shift=0, make=None):
    """(view [n, dim] whose rows are dim + pad apart and begin `shift` elements into memory, the whole memory)."""
    store = torch.full((n * (dim + pad) + shift + 16,), GUARD, dtype=dtype, device="cuda")
    view = store[shift:shift + n * (dim + pad)].view(n, dim + pad)[:, :dim]
    if make is not None:
        view.copy_(make)
    return view, store


def outside_kept(view, store, shift):
    """Nothing but the rows was written."""
    seen = store.clone()
    n, dim = view.shape
    seen[shift:shift + n * view.stride(0)].view(n, view.stride(0))[:, :dim] = GUARD
    return bool((seen == GUARD).all())


def near(got, want, off, dtype):
    bad = (got.double() - want).abs() > ref.HALF_STEP[dtype] * want.abs() * (1 + 2 ** -7) + off + torch.finfo(dtype).tiny * ref.HALF_STEP[dtype]
    assert not bool((bad | torch.isnan(got.double())).any()), (int(bad.sum()), float((got.double() - want).abs().max()))


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(*shape, seed):
    return torch.randn(*shape, device="cuda", generator=gen(seed))


# ------------------------------------------------------------------------------------------------- embedding
SHAPES = [(1, 8, 1), (5, 8, 3), (3, 1, 2), (33, 24, 8), (64, 8192, 2), (300, 257, 1), (1000, 130, 4), (17, 4099, 1)]   # n, dim, world


def ids(n, vocab, seed, absent=0.2):
    t = (torch.rand(n, device="cuda", generator=gen(seed)) ** 3 * vocab).long()
    lost = torch.rand(n, device="cuda", generator=gen(seed + 1)) < absent
    return torch.where(lost, torch.tensor([-1, vocab, -(1 << 40), 1 << 40], device="cuda")[torch.arange(n, device="cuda") % 4], t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,dim,world", SHAPES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_embedding_lookup_is_exact(dtype, n, dim, world, pad, shift):
    vocab = 40 * world
    table = [rows(40, dim, dtype, pad, shift, randn(40, dim, seed=r))[0] for r in range(world)]
    t = ids(n, vocab, n)
    whole = torch.cat(list(table))
    there = (t >= 0) & (t < vocab)
    for scale in (1.0, 0.7318):
        out, store = rows(n, dim, dtype, pad, shift + 1)
        iris.iris_embed_tokens(table, vocab, dim, KIND[dtype], t, n, out, scale=scale, shard_stride=dim + pad, out_stride=dim + pad)
        want = (whole[t.clamp(0, vocab - 1)].float() * scale).to(dtype) * there[:, None].to(dtype)
        assert torch.equal(out, want) and outside_kept(out, store, shift + 1)


def test_embedding_of_shards_that_are_not_here():
    table = randn(64, 100, seed=1)
    shards, t = list(table.chunk(4)), torch.arange(64, device="cuda")
    parts = []
    for keep in ((0, 2), (1, 3)):
        out = torch.empty(64, 100, device="cuda")
        iris.iris_embed_tokens([s if r in keep else None for r, s in enumerate(shards)], 64, 100, iris.IRIS_F32, t, 64, out)
        parts.append(out)
    assert torch.equal(parts[0] + parts[1], table)
    assert bool((parts[0][16:32] == 0).all()) and bool((parts[1][:16] == 0).all())


GRADS = [(BF16, FP32), (BF16, BF16), (FP16, FP32), (FP16, FP16), (FP32, FP32)]


def embed_grad(t, g, shards, vocab, gtype, **kw):
    n, dim = g.shape
    work = torch.empty(iris.iris_embed_workspace_bytes(n, vocab, dim), dtype=torch.uint8, device="cuda").fill_(0xA5)
    iris.iris_embed_tokens_backward(g, n, dim, KIND[g.dtype], t, shards, vocab, KIND[gtype], work, grad_out_stride=g.stride(0) if n > 1 else 0,
                                    shard_stride=shards[0].stride(0), **kw)


@pytest.mark.parametrize("dtype,gtype", GRADS)
@pytest.mark.parametrize("n,dim,world", SHAPES + [(5000, 72, 2), (9001, 515, 1)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_gradient(dtype, gtype, n, dim, world, pad, shift, accumulate):
    """Whole numbers, whose 32-bit sums are exact: one rounding to the gradient's type is left."""
    vocab = 24 * world
    t = ids(n, vocab, n + 5)
    g, _ = rows(n, dim, dtype, pad, shift, torch.randint(-8, 9, (n, dim), device="cuda", generator=gen(n)).float())
    old = torch.randint(-8, 9, (vocab, dim), device="cuda", generator=gen(n + 1)).float()
    shards = [rows(24, dim, gtype, pad, shift, old[24 * r:24 * r + 24]) for r in range(world)]
    embed_grad(t, g, [s for s, _ in shards], vocab, gtype, scale=0.5, accumulate=accumulate)
    want, _ = ref.embed_grad(t, g, vocab, 0.5)
    if accumulate:
        want += old.double()
    for r, (s, store) in enumerate(shards):
        assert torch.equal(s, want[24 * r:24 * r + 24].to(gtype)) and outside_kept(s, store, shift)


@pytest.mark.parametrize("what", ["one token", "two tokens", "all different", "none", "rising", "last"])
@pytest.mark.parametrize("n", [1, 31, 33, 1000, 4096, 4097, 20011])
def test_embedding_gradient_of_runs(what, n):
    """Runs of equal tokens of every length, over chunks and blocks; a table with more bits than one or two digits."""
    vocab = {"all different": 32768, "rising": 1 << 11, "last": (1 << 21) + 1}.get(what, 4096)
    place = torch.arange(n, device="cuda")
    t = {"one token": place * 0 + 4095, "two tokens": torch.where(place % 3 == 0, 7, 4000), "all different": place.flip(0) * 1 % 32768, "none": place * 0 - 1,
         "rising": place // 11 % (1 << 11), "last": (1 << 21) - place % 5 * 1024}[what]
    dim = 8
    g = torch.randint(-8, 9, (n, dim), device="cuda", generator=gen(n)).bfloat16()
    grad = torch.full((vocab, dim), GUARD, device="cuda")
    embed_grad(t, g, [grad], vocab, FP32)
    assert torch.equal(grad.double(), ref.embed_grad(t, g, vocab, 1.0)[0])


def test_embedding_gradient_rounds_once():
    """Sums of many terms stay within a few roundings of 32 bits: chains of 256, then of at most n / 256 / 8 + 8 sums."""
    n, vocab, dim = 30000, 50, 256
    t = ids(n, vocab, 3)
    g = torch.rand(n, dim, device="cuda", generator=gen(4)).bfloat16()
    grad = torch.empty(vocab, dim, device="cuda")
    embed_grad(t, g, [grad], vocab, FP32, scale=3.0)
    want, size = ref.embed_grad(t, g, vocab, 3.0)
    near(grad, want, (256 + n / 256 / 8 + 8 + 1) * ref.F32 * size, FP32)


def test_embedding_gradient_is_the_same_every_time():
    n, vocab, dim = 9000, 300, 333
    t, g = ids(n, vocab, 3), randn(9000, 333, seed=5).half()
    out = [torch.empty(vocab, dim, device="cuda") for _ in range(4)]
    for o in out:
        embed_grad(t, g, [o], vocab, FP32)
    assert all(torch.equal(out[0], o) for o in out[1:])


def test_embedding_gradient_of_shards_that_are_not_here():
    t, g = torch.arange(50, device="cuda") % 40, randn(50, 64, seed=3)
    shards = [torch.full((10, 64), GUARD, device="cuda") for _ in range(4)]
    embed_grad(t, g, [shards[0], None, None, shards[3]], 40, FP32)
    want, _ = ref.embed_grad(t, g, 40, 1.0)
    near(torch.cat([shards[0], shards[3]]), torch.cat([want[:10], want[30:]]), 8 * ref.F32, FP32)


def test_embedding_of_nothing():
    grad = torch.full((8, 16), GUARD, device="cuda")
    none = torch.empty(0, 16, device="cuda")
    embed_grad(torch.empty(0, dtype=torch.int64, device="cuda"), none, [grad], 8, FP32, accumulate=True)
    assert bool((grad == GUARD).all())
    embed_grad(torch.empty(0, dtype=torch.int64, device="cuda"), none, [grad], 8, FP32)
    assert bool((grad == 0).all())
    iris.iris_embed_tokens([grad], 8, 16, iris.IRIS_F32, None, 0, none)


# ------------------------------------------------------------------------------------------------- layer norm
NORMS = [(1, 1), (3, 2), (2, 8), (5, 100), (40, 128), (9, 256), (33, 1000), (7, 1025), (700, 300), (6, 2563), (5, 4096), (3, 8192), (2, 16384), (2, 16385),
         (3, 40001), (2, 65536)]


def norm_inputs(n, dim, dtype, ptype, pad, shift, offset=0.0):
    x, _ = rows(n, dim, dtype, pad, shift, randn(n, dim, seed=n + dim) * torch.exp(randn(dim, seed=dim)) + offset)
    w, b = ((1 + 0.3 * randn(dim, seed=3)).to(ptype), randn(dim, seed=4).to(ptype))
    return x, w, b


@pytest.mark.parametrize("dtype,ptype", GRADS)
@pytest.mark.parametrize("n,dim", NORMS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_norm(dtype, ptype, n, dim, pad, shift):
    x, w, b = norm_inputs(n, dim, dtype, ptype, pad, shift, offset=2.0)
    for weight, bias in ((w, b), (None, None), (w, None), (None, b)):
        y, store = rows(n, dim, dtype, pad + 1, shift + 1)
        stats = torch.full((n, 2), GUARD, device="cuda")
        iris.iris_layer_norm(x, n, dim, KIND[dtype], y, weight=weight, bias=bias, param_dtype=KIND[ptype], stats=stats, eps=1e-3, row_stride=dim + pad,
                             out_stride=dim + pad + 1)
        want, want_stats, off, off_stats = ref.norm(x, weight, bias, 1e-3)
        near(y, want, off, dtype)
        near(stats, want_stats, off_stats, FP32)
        assert outside_kept(y, store, shift + 1)


@pytest.mark.parametrize("dtype,ptype", GRADS)
@pytest.mark.parametrize("n,dim", NORMS)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_norm_gradient(dtype, ptype, n, dim, pad, shift):
    x, w, _ = norm_inputs(n, dim, dtype, ptype, pad, shift)
    dy, _ = rows(n, dim, dtype, pad + 8, shift, randn(n, dim, seed=8))
    stats = ref.norm(x, w, None, 1e-3)[1].float()
    for weight, wanted in ((w, "xwb"), (None, "xwb"), (w, "x"), (w, "w"), (w, "b")):
        dx, store = rows(n, dim, dtype, pad, shift + 2)
        dw, db = torch.full((2, dim), GUARD, device="cuda").to(ptype)
        work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda").fill_(0xA5)
        iris.iris_layer_norm_backward(x, n, dim, KIND[dtype], dy, stats, work if wanted != "x" else None, weight=weight, param_dtype=KIND[ptype],
                                      dx=dx if "x" in wanted else None, dweight=dw if "w" in wanted else None, dbias=db if "b" in wanted else None,
                                      row_stride=dim + pad, dy_stride=dim + pad + 8, dx_stride=dim + pad)
        want_x, want_w, want_b, off_x, off_w, off_b = ref.norm_grad(x, dy, weight, stats)
        if "x" in wanted:
            near(dx, want_x, off_x, dtype)
        if "w" in wanted:
            near(dw, want_w, off_w, ptype)
        if "b" in wanted:
            near(db, want_b, off_b, ptype)
        assert outside_kept(dx, store, shift + 2) and ("x" in wanted or bool((dx == GUARD).all()))
        assert ("w" in wanted or bool((dw == GUARD).all())) and ("b" in wanted or bool((db == GUARD).all()))


def test_norm_gradient_against_differences():
    """In the direction v: d sum(y c) = <dx, v>, by central differences of the 64-bit definition."""
    n, dim, step = 4, 96, 1e-5
    x, w, b = randn(n, dim, seed=1), randn(dim, seed=2), randn(dim, seed=3)
    c = randn(n, dim, seed=4)
    stats = ref.norm(x, w, b, 1e-2)[1].float()
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda")
    iris.iris_layer_norm_backward(x, n, dim, iris.IRIS_F32, c, stats, work, weight=w, dx=dx, dweight=dw, dbias=db)
    at = [t.double() for t in (x, w, b)]
    for i, grad in enumerate((dx, dw, db)):
        v = randn(*grad.shape, seed=9 + i).double()
        ends = [(ref.norm(*[t + s * step * v if j == i else t for j, t in enumerate(at)], 1e-2)[0] * c.double()).sum() for s in (1, -1)]
        want = (ends[0] - ends[1]) / (2 * step)
        assert abs(float((grad.double() * v).sum() - want)) < 1e-4 * (1 + abs(float(want)))   # 400 terms of 32 bits, differences to 1e-8


def test_norm_of_many_rows():
    """Sums down 70000 rows: chains of 128 of a thread's rows, and of their sums."""
    n, dim = 70000, 64
    x, dy = randn(n, dim, seed=1) + 0.5, torch.rand(n, dim, device="cuda", generator=gen(2))
    stats = ref.norm(x, None, None, 0.0)[1].float()
    dw, db = torch.empty(2, dim, device="cuda")
    work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda")
    iris.iris_layer_norm_backward(x, n, dim, iris.IRIS_F32, dy, stats, work, dweight=dw, dbias=db)
    _, want_w, want_b, _, off_w, off_b = ref.norm_grad(x, dy, None, stats)
    near(dw, want_w, off_w, FP32)
    near(db, want_b, off_b, FP32)


@pytest.mark.parametrize("n,dim,dtype,pad", [(700, 4200, BF16, 0), (600, 6001, FP16, 3), (500, 8192, FP32, 0), (700, 12008, BF16, 0), (400, 20001, BF16, 1), (310, 33000, FP16, 0),
                                             (200, 65536, FP32, 0), (20000, 4104, BF16, 0), (9700, 8200, BF16, 0)])
def test_norm_of_many_rows_of_several_blocks(n, dim, dtype, pad):
    """Clusters whose groups take several rows each, the last two cases more than a chain of 128; twice the same bits."""
    x, w, b = norm_inputs(n, dim, dtype, dtype, pad, 0, offset=1.0)
    dy, _ = rows(n, dim, dtype, pad, 0, torch.rand(n, dim, device="cuda", generator=gen(2)) - 0.3)
    stats = torch.empty(n, 2, device="cuda")
    y, store = rows(n, dim, dtype, pad, 0)
    got = []
    for _ in range(2):
        iris.iris_layer_norm(x, n, dim, KIND[dtype], y, weight=w, bias=b, param_dtype=KIND[dtype], stats=stats, row_stride=dim + pad, out_stride=dim + pad)
        dx, dx_store = rows(n, dim, dtype, pad, 0)
        dw, db = torch.empty(2, dim, device="cuda", dtype=dtype)
        work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda").fill_(0xA5)
        iris.iris_layer_norm_backward(x, n, dim, KIND[dtype], dy, stats, work, weight=w, param_dtype=KIND[dtype], dx=dx, dweight=dw, dbias=db,
                                      row_stride=dim + pad, dy_stride=dim + pad, dx_stride=dim + pad)
        got.append([t.clone() for t in (y, stats, dx, dw, db)])
    assert all(bool((p == q).all()) for p, q in zip(*got)) and outside_kept(y, store, 0) and outside_kept(dx, dx_store, 0)
    want, want_stats, off, off_stats = ref.norm(x, w, b, 1e-5)
    near(y, want, off, dtype)
    near(stats, want_stats, off_stats, FP32)
    del want, off
    want_x, want_w, want_b, off_x, off_w, off_b = ref.norm_grad(x, dy, w, stats)
    near(dx, want_x, off_x, dtype)
    near(dw, want_w, off_w, dtype)
    near(db, want_b, off_b, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,dim,pad", [(50, 1000, 0), (9, 4097, 3), (4, 20000, 8)])
def test_norm_in_place(dtype, n, dim, pad):
    x, w, b = norm_inputs(n, dim, dtype, FP32, pad, 1)
    dy = rows(n, dim, dtype, pad, 1, randn(n, dim, seed=8))[0]
    args, s = (n, dim, KIND[dtype]), dict(row_stride=dim + pad)
    stats, y = torch.empty(n, 2, device="cuda"), rows(n, dim, dtype, pad, 1)[0]
    iris.iris_layer_norm(x, *args, y, weight=w, bias=b, stats=stats, out_stride=dim + pad, **s)
    dx = rows(n, dim, dtype, pad, 1)[0]
    iris.iris_layer_norm_backward(x, *args, dy, stats, weight=w, dx=dx, dy_stride=dim + pad, dx_stride=dim + pad, **s)
    for which in (x, dy):
        a, g = rows(n, dim, dtype, pad, 1, x)[0], rows(n, dim, dtype, pad, 1, dy)[0]
        to = a if which is x else g
        iris.iris_layer_norm_backward(a, *args, g, stats, weight=w, dx=to, dy_stride=dim + pad, dx_stride=dim + pad, **s)
        assert torch.equal(to, dx)
    iris.iris_layer_norm(x, *args, x, weight=w, bias=b, out_stride=dim + pad, **s)
    assert torch.equal(x, y)


def test_norm_rows_do_not_notice_one_another():
    x = randn(6, 3000, seed=1)
    y, clean = torch.empty_like(x), torch.empty_like(x)
    iris.iris_layer_norm(x, 6, 3000, iris.IRIS_F32, clean)
    x[1, 7], x[3, 2999], x[4] = math.nan, math.inf, 5.0
    iris.iris_layer_norm(x, 6, 3000, iris.IRIS_F32, y, eps=0.0)
    assert all(bool(torch.isnan(y[r]).all()) for r in (1, 3, 4))
    iris.iris_layer_norm(x, 6, 3000, iris.IRIS_F32, y)
    assert bool((y[4] == 0).all()) and all(torch.equal(y[r], clean[r]) for r in (0, 2, 5))


def test_norm_of_large_offsets():
    """The spread of rows far from 0 is not lost: x is exact, 1000 + small."""
    x = 1000 + torch.randint(-64, 65, (5, 2048), device="cuda", generator=gen(3)) / 64
    y = torch.empty_like(x)
    iris.iris_layer_norm(x, 5, 2048, iris.IRIS_F32, y)
    want, _, off, _ = ref.norm(x, None, None, 1e-5)
    near(y, want, off, FP32)
    assert float(off.max()) < 0.02


def test_norm_of_no_rows():
    dw, db = torch.full((2, 16), GUARD, device="cuda")
    none = torch.empty(0, 16, device="cuda")
    iris.iris_layer_norm(none, 0, 16, iris.IRIS_F32, none)
    iris.iris_layer_norm_backward(none, 0, 16, iris.IRIS_F32, none, None, dweight=dw, dbias=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


# ------------------------------------------------------------------------------------------------- verification
def verify(z, n, ids_, u, e, q=None, scale=1.0, scales=None, logprob=True, **kw):
    b, vocab = e.shape
    tokens = torch.full((b, n + 1), -7, dtype=torch.int64, device="cuda")
    accepted, lp = torch.full((b,), -7, dtype=torch.int64, device="cuda"), torch.full((b, n + 1), GUARD, device="cuda")
    work = torch.empty(iris.iris_verify_workspace_bytes(b, n), dtype=torch.uint8, device="cuda").fill_(0xA5)
    iris.iris_verify_drafts(z, b, n, vocab, KIND[z.dtype], ids_, u, e, tokens, accepted, work, draft_logits=q, logprob=lp if logprob else None, scale=scale,
                            scales=scales, row_stride=z.stride(0), draft_stride=0 if q is None else q.stride(0), **kw)
    return tokens, accepted, lp


def check_verify(z, n, ids_, u, e, q=None, scale=1.0, scales=None):
    tokens, accepted, lp = verify(z, n, ids_, u, e, q, scale, scales)
    b = e.shape[0]
    zc, qc, ic, uc, ec = (None if t is None else t.cpu() for t in (z, q, ids_, u, e))
    close = 0
    for i in range(b):
        s = scale if scales is None else float(scales[i])
        want, count, want_lp, margin = ref.verify(zc[i * (n + 1):(i + 1) * (n + 1)], None if q is None else qc[i * n:(i + 1) * n], ic[i], uc[i], ec[i],
                                                  float(torch.tensor(s, dtype=torch.float32)))
        if margin < 2.0 ** -16:   # within 32-bit arithmetic of another outcome
            close += 1
            continue
        assert tokens[i].tolist() == want and int(accepted[i]) == count, (i, tokens[i].tolist(), want, margin)
        for got, w in zip(lp[i].tolist(), want_lp):
            # sums of 32 bits are off by 2^-20, the result is rounded once
            assert got == w or abs(got - w) <= 2.0 ** -20 + 2.0 ** -23 * abs(w), (i, got, w)
    assert close <= max(1, b // 8)


def drafted(b, n, vocab, dtype, seed, pad=0, shift=0, with_q=True, ragged=False, masked=0.0, agree=0.5, soft=1.0):
    z = randn(b * (n + 1), vocab, seed=seed) * 2
    if masked:
        z.masked_fill_(torch.rand(z.shape, device="cuda", generator=gen(seed + 5)) < masked, -math.inf)
    near_z = z.view(b, n + 1, vocab)[:, :n].reshape(b * n, vocab)
    y = (near_z + agree * randn(b * n, vocab, seed=seed + 1)).to(dtype)
    z = rows(b * (n + 1), vocab, dtype, pad, shift, z)[0]
    race = torch.empty(b * n, vocab, device="cuda").exponential_(generator=gen(seed + 2))
    t = (y.float() * soft - race.log()).argmax(1).view(b, n) if n else torch.empty(b, 0, dtype=torch.int64, device="cuda")
    if ragged and n:
        t = torch.where(torch.arange(n, device="cuda") < torch.randint(0, n + 1, (b, 1), device="cuda", generator=gen(seed + 3)), t, -1)
    u = torch.rand(b, n, device="cuda", generator=gen(seed + 4))
    e = torch.empty(b, vocab, device="cuda").exponential_(generator=gen(seed + 6))
    return z, t, u, e, rows(b * n, vocab, dtype, pad, shift + 1, y)[0] if with_q and n else None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,n,vocab", [(1, 0, 1), (3, 2, 1), (4, 1, 7), (16, 3, 100), (9, 8, 1000), (2, 40, 515), (3, 4, 20011), (1, 3, 70000), (40, 0, 4096)])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_verify(dtype, b, n, vocab, pad, shift):
    for with_q, ragged, masked in ((True, False, 0.0), (True, True, 0.5), (False, False, 0.0), (False, True, 0.7)):
        z, t, u, e, q = drafted(b, n, vocab, dtype, b + n + vocab, pad, shift, with_q, ragged, masked if vocab > 7 else 0.0)
        check_verify(z, n, t, u, e, q, scale=0.8)


@pytest.mark.parametrize("dtype", TYPES)
def test_verify_with_a_scale_for_each_sequence(dtype):
    b, n, vocab = 24, 4, 3001
    z, t, u, e, q = drafted(b, n, vocab, dtype, 5, with_q=True, agree=0.3)
    scales = torch.rand(b, device="cuda", generator=gen(1)) * 2 + 0.2
    scales[::3] = math.inf
    best = z.view(b, n + 1, vocab)[:, :n].float().argmax(2)
    t[::6] = best[::6]           # greedy and right
    t[9, :2] = best[9, :2]       # right for two places
    check_verify(z, n, t, u, e, q, scales=scales)
    check_verify(z, n, best, u, e, None, scale=math.inf)
    tokens, accepted, lp = verify(z, n, best, u, e, None, scale=math.inf)
    assert bool((accepted == n).all()) and bool((lp == 0).all())


def test_verify_greedy_takes_the_lowest_of_equal_logits():
    for dtype in TYPES:
        for vocab, shift in ((50, 3), (5003, 1), (40009, 0)):
            z, _ = rows(4, vocab, dtype, 0, shift, torch.zeros(4, vocab, device="cuda"))
            z[0, 5:] = 3.0
            z[1, vocab - 1] = 3.0
            z[2, 0] = z[2, 9] = z[2, vocab - 2] = 3.0
            z[3] = -math.inf
            none = torch.empty(4, 0, device="cuda")
            tokens, _, _ = verify(z, 0, none.long(), none, torch.ones(4, vocab, device="cuda"), scale=math.inf)
            assert tokens[:, 0].tolist() == [5, vocab - 1, 0, -1]


def test_verify_rows_without_a_distribution():
    """Empty rows, NaN and +inf, of the target and of the draft; a lowest finite mask; a row of one token."""
    vocab, n, b = 900, 2, 9
    z, t, u, e, q = drafted(b, n, vocab, FP32, 3)
    t[:] = 5
    z[:, 5] = 6.0
    q[:, 5] = 5.0
    u[:] = 0.01
    z[0 * 3] = -math.inf
    z[1 * 3 + 1, 800] = math.nan
    z[2 * 3 + 2, 3] = math.inf
    q[3 * 2] = -math.inf            # q(d) = 0 < p(d): accepted
    q[4 * 2 + 1, 7] = math.nan
    q[5 * 2, 7] = math.inf
    z[6 * 3] = torch.finfo(FP32).min
    z[7 * 3] = -math.inf
    z[7 * 3, 5] = -2.0
    z[8 * 3] = -math.inf
    z[8 * 3, 6] = -2.0              # all but one masked, and the draft names another
    check_verify(z, n, t, u, e, q)
    tokens, accepted, lp = verify(z, n, t, u, e, q)
    assert accepted[:6].tolist() == [0, 1, 2, 2, 1, 0] and accepted[7:].tolist() == [2, 0]
    assert tokens[0].tolist() == [-1] * 3 and tokens[1].tolist() == [5, -1, -1] and tokens[2].tolist() == [5, 5, -1]
    assert tokens[8].tolist() == [6, -1, -1] and float(lp[8, 0]) == 0.0
    bad = torch.tensor([math.nan, 0.0, -1.0, -math.inf, 1.0, 1.0, 1.0, 1.0, 1.0], device="cuda")
    tokens, accepted, lp = verify(z, n, t, u, e, q, scales=bad)
    assert accepted[:4].tolist() == [0] * 4 and bool((tokens[:4] == -1).all()) and bool((lp[:4] == 0).all())


def test_verify_noise_that_is_not_positive():
    z = torch.zeros(5, 64, device="cuda")
    e = torch.ones(5, 64, device="cuda")
    e[0, 3:], e[1, 40], e[2, 10:13], e[3], e[4] = -1.0, 0.0, 0.0, math.nan, math.inf
    e[0, :3] = torch.tensor([3.0, 0.5, 2.0])
    none = torch.empty(5, 0, device="cuda")
    tokens, _, _ = verify(z, 0, none.long(), none, e)
    assert tokens[:, 0].tolist() == [1, 40, 10, -1, -1]


def test_verify_a_draft_that_is_the_target_is_always_accepted():
    b, n, vocab = 30, 5, 2000
    z, t, u, e, _ = drafted(b, n, vocab, BF16, 2)
    q = z.view(b, n + 1, vocab)[:, :n].reshape(b * n, vocab).clone()
    u[:] = 1 - 2.0 ** -24
    tokens, accepted, _ = verify(z, n, t, u, e, q)
    assert bool((accepted == n).all()) and torch.equal(tokens[:, :n], t)


def test_verify_draws_as_the_target_would():
    """20000 sequences of one context: accepted and redrawn tokens together are distributed as p.  The counts' chi-squared over 15 degrees of freedom
    has mean 15 and variance 30: above 60 with a probability below 1e-6."""
    b, vocab = 20000, 16
    zt, zq = randn(2, vocab, seed=1).repeat(b, 1), randn(1, vocab, seed=2).repeat(b, 1)
    race = torch.empty(b, vocab, device="cuda").exponential_(generator=gen(3))
    t = (zq - race.log()).argmax(1)[:, None]
    u, e = torch.rand(b, 1, device="cuda", generator=gen(4)), torch.empty(b, vocab, device="cuda").exponential_(generator=gen(5))
    tokens, accepted, _ = verify(zt, 1, t, u, e, zq)
    for place, row, seen in ((0, zt[0], tokens[:, 0]), (1, zt[1], tokens[:, 1][accepted == 1])):
        want = torch.softmax(row.double(), 0) * seen.shape[0]
        got = torch.bincount(seen, minlength=vocab).double()
        assert float(((got - want) ** 2 / want).sum()) < 60, place
    assert 0.2 < float(accepted.double().mean()) < 0.95


def test_verify_is_the_same_every_time_and_for_each_sequence_alone():
    b, n, vocab = 12, 3, 30011
    z, t, u, e, q = drafted(b, n, vocab, FP16, 4, pad=3, shift=1)
    first = verify(z, n, t, u, e, q)
    again = verify(z, n, t, u, e, q)
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    for i in range(b):
        one = verify(z[i * (n + 1):(i + 1) * (n + 1)], n, t[i:i + 1], u[i:i + 1], e[i:i + 1], q[i * n:(i + 1) * n])
        assert torch.equal(one[0][0], first[0][i]) and int(one[1]) == int(first[1][i])
