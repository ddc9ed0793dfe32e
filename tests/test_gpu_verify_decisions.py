"""Verification of drafts where 32 bits cannot tell: rows without a distribution."""
import math

import pytest
import torch

from test_gpu_head_ops import TYPES, check_verify, drafted, verify

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
