"""The limit on the waits of blocks that share a norm's rows: a wait that runs out is recorded and gives NaN, the call ends, and calls after it are right."""
import pytest
import torch

import paper_2511_12500_b200 as iris
import head_ref as ref
from test_gpu_head_ops import BF16, FP32, GUARD, KIND, near, outside_kept, randn, rows

pytestmark = pytest.mark.gpu


@pytest.fixture
def withhold():
    """Called with True: blocks keep their sums to themselves."""
    iris.iris_layer_norm_status()
    yield iris.iris_layer_norm_withhold
    iris.iris_layer_norm_withhold(False)


def timed_out(call):
    call()
    with pytest.raises(iris.IrisError) as e:
        iris.iris_layer_norm_status()
    assert e.value.code == iris.IRIS_ERR_TIMEOUT and e.value.detail[:2] == [iris.IRIS_ERR_TIMEOUT, 5], e.value.detail
    iris.iris_layer_norm_status()   # cleared


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("dim,pad,shift", [(16384, 0, 0), (30003, 3, 1)])
def test_a_wait_that_runs_out(withhold, dtype, dim, pad, shift):
    n = 400
    x, _ = rows(n, dim, dtype, pad, shift, randn(n, dim, seed=1))
    dy, _ = rows(n, dim, dtype, pad, shift, randn(n, dim, seed=2))
    y, y_store = rows(n, dim, dtype, pad, shift)
    dx, dx_store = rows(n, dim, dtype, pad, shift)
    stats, dw, db = torch.empty(n, 2, device="cuda"), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    work = torch.empty(iris.iris_layer_norm_workspace_bytes(n, dim), dtype=torch.uint8, device="cuda")
    at = dict(row_stride=dim + pad)

    def forward():
        iris.iris_layer_norm(x, n, dim, KIND[dtype], y, stats=stats, out_stride=dim + pad, **at)

    def backward():
        iris.iris_layer_norm_backward(x, n, dim, KIND[dtype], dy, stats, work, dx=dx, dweight=dw, dbias=db, dy_stride=dim + pad, dx_stride=dim + pad, **at)

    withhold(True)
    timed_out(forward)
    assert bool(torch.isnan(y).any()) and bool(torch.isnan(stats).any()) and outside_kept(y, y_store, shift)
    withhold(False)
    forward()
    iris.iris_layer_norm_status()
    want, want_stats, off, off_stats = ref.norm(x, None, None, 1e-5)
    near(y, want, off, dtype)
    withhold(True)
    timed_out(backward)
    assert bool(torch.isnan(dx).any()) and outside_kept(dx, dx_store, shift)
    want, want_dw, want_db, off, off_dw, off_db = ref.norm_grad(x, dy, None, stats)
    near(dw, want_dw, off_dw, FP32)
    near(db, want_db, off_db, FP32)
    withhold(False)
    backward()
    iris.iris_layer_norm_status()
    near(dx, want, off, dtype)
    near(dw, want_dw, off_dw, FP32)


def test_rows_of_one_block_wait_for_nobody(withhold):
    withhold(True)
    x = randn(300, 8192, seed=1)
    y = torch.full_like(x, GUARD)
    iris.iris_layer_norm(x, 300, 8192, iris.IRIS_F32, y)
    iris.iris_layer_norm_status()
    want, _, off, _ = ref.norm(x, None, None, 1e-5)
    near(y, want, off, FP32)
