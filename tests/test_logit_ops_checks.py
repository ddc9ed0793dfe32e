"""More of what the operators on logits refuse before anything is launched (no GPU needed): scales whose exponents overflow, and
tensors that are not what the call takes them for."""
import numpy as np
import pytest
import torch

import paper_2511_12500_b200 as iris
from paper_2511_12500_b200 import binding, build as iris_build
from test_logit_ops_args import CALLS, P, SCORE


@pytest.fixture(scope="module", autouse=True)
def library():
    iris_build.build()


@pytest.mark.parametrize("call", sorted(CALLS))
def test_scales_whose_exponents_overflow(call):
    with pytest.raises(iris.IrisError) as e:
        getattr(iris, call)(**{**CALLS[call], "scale": 2.5e38})
    assert e.value.code == iris.IRIS_ERR_ARG and "scale is at most 2e+38" in str(e.value)


ROWS, VOCAB = SCORE["rows"], SCORE["vocab"]
# name -> (element type, elements of a row) as the calls above need them
BUFFERS = {
    "iris_token_logprobs": dict(targets=(torch.int64, 1), logprob=(torch.float32, 1), entropy=(torch.float32, 1), stats=(torch.float32, 2),
                                top_ids=(torch.int64, 5), top_logprob=(torch.float32, 5)),
    "iris_token_logprobs_backward": dict(targets=(torch.int64, 1), stats=(torch.float32, 2), grad_logprob=(torch.float32, 1), entropy=(torch.float32, 1),
                                         grad_entropy=(torch.float32, 1)),
    "iris_distill_topk": dict(teacher=(torch.float32, 8), teacher_ids=(torch.int64, 8), weight=(torch.float32, 1), loss=(torch.float32, 1),
                              stats=(torch.float32, 3)),
    "iris_distill_topk_backward": dict(teacher=(torch.float32, 8), teacher_ids=(torch.int64, 8), grad_loss=(torch.float32, 1), stats=(torch.float32, 3)),
}
WRONG_TYPE = {torch.int64: (torch.int32, torch.float64), torch.float32: (torch.float64, torch.bfloat16, torch.int32)}


def refused(call, says, **change):
    with pytest.raises(iris.IrisError) as e:
        getattr(iris, call)(**{**CALLS[call], **change})
    assert e.value.code == iris.IRIS_ERR_ARG and says in str(e.value), str(e.value)


@pytest.mark.parametrize("call,name", [(c, n) for c in BUFFERS for n in BUFFERS[c]])
def test_buffers_that_are_not_what_the_call_needs(call, name):
    """32-bit ids read as 64-bit ones, a gradient expanded from one value, a column of a wider tensor, too few elements: read past their end."""
    dtype, each = BUFFERS[call][name]
    for wrong in WRONG_TYPE[dtype]:
        refused(call, f"{name} is {wrong}, not {dtype}", **{name: torch.zeros(ROWS * each * 2, dtype=wrong)})
    refused(call, f"{name} is not contiguous", **{name: torch.zeros(1, dtype=dtype).expand(ROWS * each)})
    refused(call, f"{name} is not contiguous", **{name: torch.zeros(ROWS, each + 1, dtype=dtype)[:, :each]})
    refused(call, f"{name} has {ROWS * each - 1} elements", **{name: torch.zeros(ROWS * each - 1, dtype=dtype)})
    refused(call, f"{name} is a ndarray", **{name: np.zeros(ROWS * each, np.int64 if dtype is torch.int64 else np.float32)})
    refused(call, f"{name} is not on the GPU", **{name: torch.zeros(ROWS, each, dtype=dtype)})


@pytest.mark.parametrize("call,name,stride", [(c, n, s) for c in CALLS for n, s in (("logits", "row_stride"), ("dlogits", "grad_stride"))
                                              if n in CALLS[c] or (c, n) == ("iris_distill_topk", "dlogits")])
def test_rows_that_are_not_what_the_call_needs(call, name, stride):
    bf16 = dict(dtype=torch.bfloat16)
    refused(call, f"{name} is torch.float16, not torch.bfloat16", **{name: torch.zeros(ROWS, VOCAB, dtype=torch.float16)})
    refused(call, "the row stride is not given", **{name: torch.zeros(ROWS, VOCAB + 24, **bf16)[:, :VOCAB]})
    refused(call, "the row stride is not given", **{name: torch.zeros(ROWS, VOCAB + 24, **bf16)})
    refused(call, "the row stride is not given", **{name: torch.zeros(2 * ROWS, VOCAB, **bf16)[::2]})
    refused(call, "elements apart", **{name: torch.zeros(VOCAB, ROWS, **bf16).t(), stride: VOCAB})
    refused(call, "does not hold", **{name: torch.zeros(ROWS - 1, VOCAB, **bf16)})
    refused(call, "does not hold", **{name: torch.zeros(ROWS, VOCAB, **bf16), stride: VOCAB + 1})
    refused(call, "does not hold", **{name: torch.zeros(ROWS, VOCAB + 24, **bf16)[1:, :VOCAB], stride: VOCAB + 24})
    refused(call, "does not hold", **{name: torch.zeros(1, VOCAB, **bf16).expand(ROWS, VOCAB), stride: VOCAB})
    for right in (torch.zeros(ROWS, VOCAB, **bf16), torch.zeros(2, ROWS // 2, VOCAB, **bf16), torch.zeros(ROWS * VOCAB, **bf16)):
        refused(call, f"{name} is not on the GPU", **{name: right})
    refused(call, f"{name} is not on the GPU", **{name: torch.zeros(ROWS, VOCAB + 24, **bf16)[:, 3:VOCAB + 3], stride: VOCAB + 24})


def test_what_is_not_read_is_not_looked_at():
    binding._first_call()
    none = torch.zeros(0, dtype=torch.int32)
    look = (0, VOCAB, iris.IRIS_BF16, torch.zeros(0, VOCAB), 0, None, 0, none, 8, 1, None, 4, 1, 5, 4, 1)
    assert binding._look(("targets", "logprob", "entropy"), *look)[1:] == [0, 0, 0, 5]
    assert binding._accept(*look) in (None, (0, 0, 0, 0, 5))


def test_the_extension_is_built_and_reads_this_torch():
    """Right tensors pass without a question in Python.  (Where they are is all that it can say here: not on a GPU.)"""
    binding._first_call()
    assert binding._accept.__self__.__name__ == "paper_2511_12500_b200._tensors"
    assert binding._accept(3, 50, iris.IRIS_F32, P, 0, P + 4, 64, None, 8, 1, P, 4, 2) == (P, P + 4, 0, P)
    assert binding._accept(3, 50, iris.IRIS_F32, torch.zeros(3, 50), 0, None, 0) is None
    assert binding._accept(3, 50, iris.IRIS_F32, -1, 0, None, 0) is None and binding._accept(3, 50, iris.IRIS_F32, "x", 0, None, 0) is None
    for bad in ((), (1, 2, 3), (3, 50, 2, P, 0, None, 0, P), ("a", 50, 2, P, 0, None, 0), (3, 50, 2, P, None, None, 0), (1 << 70, 50, 2, P, 0, None, 0)):
        assert binding._accept(*bad) is None
