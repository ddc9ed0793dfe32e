"""Verification of drafts where 32 bits cannot tell: rows without a distribution, target and draft alike, runners of a race next to one another."""
import math

import pytest
import torch

from test_gpu_head_ops import BF16, FP16, FP32, TYPES, check_verify, drafted, gen, randn, rows, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [900, 70001])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("draw", [0.0, 0.01])
def test_a_draft_row_without_a_distribution_rejects_a_masked_draft(dtype, vocab, bad, draw):
    """q(d) of a masked draft is 0 in a row that has a distribution (accepted, as p(d) > 0), and unknown in one that has none (rejected)."""
    b, n = 8, 2
    z, t, u, e, q = drafted(b, n, vocab, dtype, 11, pad=3, shift=1)
    t[:], u[:] = 5, draw
    z[:, 5], q[:, 5] = 6.0, -math.inf
    q[::4, vocab // 2] = bad            # the first place of every second sequence
    check_verify(z, n, t, u, e, q)
    _, accepted, _ = verify(z, n, t, u, e, q)
    assert accepted.tolist() == [0, 2] * 4


def alike(b, n, vocab, dtype, seed, pad, shift, draft_pad, draft_shift):
    """Target and draft the same, and drafts that both mask: refused, and nothing is left of p - q."""
    x = randn(b * (n + 1), vocab, seed=seed) * 3
    t = torch.randint(0, vocab, (b, n), device="cuda", generator=gen(seed + 1))
    x.view(b, n + 1, vocab)[:, :n].scatter_(2, t[:, :, None], -math.inf)
    z = rows(b * (n + 1), vocab, dtype, pad, shift, x)[0]
    q = rows(b * n, vocab, dtype, draft_pad, draft_shift, x.view(b, n + 1, vocab)[:, :n].reshape(b * n, vocab))[0]
    return z, t, torch.zeros(b, n, device="cuda"), torch.empty(b, vocab, device="cuda").exponential_(generator=gen(seed + 2)), q


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("b,n,vocab", [(40, 1, 1000), (300, 2, 77), (9, 3, 20011), (2, 2, 128000), (1, 1, 128003)])
@pytest.mark.parametrize("lie", [(0, 0, 0, 0), (8, 0, 0, 0), (3, 1, 3, 1), (0, 0, 5, 3), (1, 2, 0, 1)])   # pad, shift of the target's rows and of the draft's
def test_target_and_draft_alike_leave_the_target(dtype, b, n, vocab, lie):
    z, t, u, e, q = alike(b, n, vocab, dtype, b + vocab, *lie)
    for scale in (1.0, 0.37):
        check_verify(z, n, t, u, e, q, scale=scale)
        tokens, accepted, _ = verify(z, n, t, u, e, q, scale=scale)
        assert bool((accepted == 0).all()) and bool((tokens[:, 0] >= 0).all())
    e[:, 7::50] = 0.0                   # the first of them that is not masked wins
    check_verify(z, n, t, u, e, q)


def test_target_and_draft_alike_draw_as_the_target_would():
    """20000 sequences of one context.  The counts' chi-squared over 14 degrees of freedom has mean 14 and variance 28: above 60 with a probability below 1e-6."""
    b, vocab = 20000, 16
    z = randn(1, vocab, seed=1)
    z[0, 3] = -math.inf
    e = torch.empty(b, vocab, device="cuda").exponential_(generator=gen(5))
    t, u = torch.full((b, 1), 3, device="cuda"), torch.zeros(b, 1, device="cuda")
    tokens, accepted, _ = verify(z.repeat(2 * b, 1), 1, t, u, e, z.repeat(b, 1))
    assert bool((accepted == 0).all())
    want = torch.softmax(z[0].double(), 0) * b
    got = torch.bincount(tokens[:, 0], minlength=vocab).double()
    keep = want > 0
    assert float(got[3]) == 0 and float(((got - want)[keep] ** 2 / want[keep]).sum()) < 60


def first_of_largest(score):
    """(column of the largest score, the lowest of equal ones; by how much it is ahead of the next different one, relative)."""
    best = score.amax(1, keepdim=True)
    columns = torch.arange(score.shape[1], device="cuda")
    at = torch.where(score == best, columns, score.shape[1]).amin(1)
    rest = torch.where(score == best, -math.inf, score).amax(1)
    return at, (best[:, 0] - rest) / best[:, 0]


def next_to(x, steps):
    """fp32 numbers `steps` further (x > 0)."""
    return (x.view(torch.int32) + steps).view(torch.float32)


# 64-bit scores of one row: an exponential, a quotient and a product, each off by 2^-52 or so, of numbers below 2^7 times their scale
NEAR = 2.0 ** -44


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("apart", [1, 3, 1024, 2048, 4096, 8192, 17011])   # in a thread's 16 bytes, in one thread's, in two threads', in two blocks'
@pytest.mark.parametrize("b", [200, 4])
def test_runners_next_to_one_another(dtype, apart, b):
    """Two tokens whose scores p / e are the same but for the last bits of their noise: the sum of p does not matter, so 64 bits tell which is ahead."""
    vocab, scale, rounds = 40000, 0.75, 200 // b
    for k in range(rounds):
        z = rows(b, vocab, dtype, 3, 1, randn(b, vocab, seed=k) * 2)[0]
        a = torch.randint(0, vocab - apart, (b, 1), device="cuda", generator=gen(k + 1))
        za, zb = z.gather(1, a).double(), z.gather(1, a + apart).double()
        ea = torch.rand(b, 1, device="cuda", generator=gen(k + 2)) * 1.5 + 0.5
        eb = next_to((ea.double() * ((zb - za) * scale).exp()).float(), torch.randint(-2, 3, (b, 1), device="cuda", generator=gen(k + 3), dtype=torch.int32))
        e = torch.full((b, vocab), 1e9, device="cuda").scatter_(1, a, ea).scatter_(1, a + apart, eb)
        want, ahead = first_of_largest(((z.double() - z.double().amax(1, keepdim=True)) * scale).exp() / e.double())
        none = torch.empty(b, 0, device="cuda")
        tokens, _, _ = verify(z, 0, none.long(), none, e, scale=scale)
        wrong = (tokens[:, 0] != want) & (ahead > NEAR)
        assert not bool(wrong.any()), (int(wrong.sum()), float(ahead[wrong].max()))
        assert int((ahead > NEAR).sum()) >= b - max(2, b // 20)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("apart", [1, 1024, 2048, 17011])
def test_equal_runners_the_lowest_column_wins(dtype, apart):
    b, vocab = 100, 40000
    z = rows(b, vocab, dtype, 3, 1, randn(b, vocab, seed=1) * 2)[0]
    a = torch.randint(0, vocab - 2 * apart, (b, 1), device="cuda", generator=gen(2))
    e = torch.full((b, vocab), 1e9, device="cuda")
    for i in range(3):
        z.scatter_(1, a + i * apart, z.gather(1, a))
        e.scatter_(1, a + i * apart, torch.rand(b, 1, device="cuda", generator=gen(3)) + 0.5)
    none = torch.empty(b, 0, device="cuda")
    tokens, _, _ = verify(z, 0, none.long(), none, e)
    assert torch.equal(tokens[:, 0], a[:, 0])


@pytest.mark.parametrize("dtype,less", [(FP32, 1e-2), (FP32, 1e-4), (FP32, 2e-5), (FP16, 2.0 ** -5), (BF16, 2.0 ** -2)])
@pytest.mark.parametrize("apart", [1, 1024, 2048, 17011])
def test_runners_of_what_a_draft_close_to_the_target_leaves(dtype, less, apart):
    """p and q are 1 - e^-40 at one token, where nothing is left; of two others with p near e^-40 a small part is.  The rows' sums are 1 in any arithmetic, so
    that 64 bits tell which of the two is ahead, and what 32 bits make of the exponentials (off by 2^-18) does not matter."""
    b, vocab = 400, 40000
    a = torch.randint(1, vocab - apart - 1, (b, 1), device="cuda", generator=gen(1))
    at = torch.cat([a, a + apart], 1)
    # each token's own: -36 .. -44, and so much less in the draft
    x = -40 + 4 * (2 * torch.rand(b, 2, device="cuda", generator=gen(2)) - 1)
    za = x.to(dtype)
    ya = (za.double() - less).to(dtype)
    assert bool((ya < za).all())
    z = torch.full((2 * b, vocab), -math.inf, device="cuda", dtype=dtype)
    z[:, 0] = 0.0
    z[::2].scatter_(1, at, za)
    q = torch.full((b, vocab), -math.inf, device="cuda", dtype=dtype)
    q[:, 0] = 0.0
    q.scatter_(1, at, ya)
    t = torch.full((b, 1), vocab - 1, device="cuda")   # masked in both
    w = za.double().exp() - ya.double().exp()
    ea = torch.rand(b, 1, device="cuda", generator=gen(3)) + 0.5
    by = 1 + (10 ** (-3.3 - 6 * torch.rand(b, 1, device="cuda", generator=gen(4), dtype=torch.float64))) * torch.randn(b, 1, device="cuda", generator=gen(5)).sign()
    eb = (ea.double() * (w[:, 1:] / w[:, :1]) * by).float()
    e = torch.ones(b, vocab, device="cuda").scatter_(1, a, ea).scatter_(1, a + apart, eb)
    score = w / torch.cat([ea, eb], 1).double()
    want = torch.where(score[:, 0] >= score[:, 1], at[:, 0], at[:, 1])
    ahead = (score[:, 0] - score[:, 1]).abs() / score.amax(1)
    tokens, accepted, _ = verify(z, 1, t, torch.zeros(b, 1, device="cuda"), e, q)
    assert bool((accepted == 0).all())
    close = NEAR / less                # 64 bits of p, of which `less` is left
    wrong = (tokens[:, 0] != want) & (ahead > close)
    assert not bool(wrong.any()), (int(wrong.sum()), float(ahead[wrong].max()))
    assert int((ahead > close).sum()) >= b - b // 20
