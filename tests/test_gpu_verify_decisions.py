"""Verification of drafts where 32 bits cannot tell: rows without a distribution, target and draft alike."""
import math

import pytest
import torch

from test_gpu_head_ops import TYPES, check_verify, drafted, gen, randn, rows, verify

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
