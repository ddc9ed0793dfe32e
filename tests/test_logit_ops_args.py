"""What the operators on logits refuse, before anything is launched (no GPU needed)."""
import ctypes

import pytest

import paper_2511_12500_b200 as iris
from paper_2511_12500_b200 import build as iris_build

P = 1 << 20   # an address that nothing reads: every call here is refused first


@pytest.fixture(scope="module", autouse=True)
def library():
    iris_build.build()


SCORE = dict(logits=P, rows=4, vocab=1000, dtype=iris.IRIS_BF16, targets=P, n_targets=1, logprob=P, entropy=P, stats=P, top_k=5, top_ids=P, top_logprob=P,
             stream=0)
SCORE_GRAD = dict(logits=P, rows=4, vocab=1000, dtype=iris.IRIS_BF16, targets=P, n_targets=1, stats=P, grad_logprob=P, dlogits=P, stream=0)
DISTILL = dict(logits=P, rows=4, vocab=1000, dtype=iris.IRIS_BF16, teacher=P, teacher_ids=P, list_k=8, loss=P, stream=0)
DISTILL_GRAD = dict(logits=P, rows=4, vocab=1000, dtype=iris.IRIS_BF16, teacher=P, teacher_ids=P, list_k=8, stats=P, grad_loss=P, dlogits=P, stream=0)
CALLS = {"iris_token_logprobs": SCORE, "iris_token_logprobs_backward": SCORE_GRAD, "iris_distill_topk": DISTILL, "iris_distill_topk_backward": DISTILL_GRAD}

COMMON = [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(vocab=-5), "vocab"), (dict(row_stride=999), "row stride"),
    (dict(row_stride=-1), "row stride"), (dict(row_stride=1 << 61), "too large"), (dict(logits=None), "logits is NULL"), (dict(logits=P + 1), "aligned"),
    (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"),
]
OWN = {
    "iris_token_logprobs": [
        (dict(n_targets=129), "n_targets"), (dict(n_targets=-1), "n_targets"), (dict(targets=None), "targets is NULL"), (dict(targets=P + 4), "targets"),
        (dict(logprob=None), "logprob is NULL"), (dict(logprob=P + 2), "logprob"), (dict(top_k=129), "top_k"), (dict(top_k=-1), "top_k"),
        (dict(vocab=4), "exceeds vocab"), (dict(top_ids=None), "top_ids is NULL"), (dict(top_ids=P + 4), "top_ids"), (dict(top_logprob=P + 1), "top_logprob"),
        (dict(entropy=P + 2), "entropy"), (dict(stats=P + 2), "stats"),
    ],
    "iris_token_logprobs_backward": [
        (dict(n_targets=129), "n_targets"), (dict(targets=None), "targets is NULL"), (dict(stats=None), "stats is NULL"), (dict(grad_entropy=P), "entropy is NULL"),
        (dict(grad_logprob=P + 2), "grad_logprob"), (dict(dlogits=None), "dlogits is NULL"), (dict(dlogits=P + 1), "aligned"), (dict(grad_stride=999), "row stride"),
        (dict(dlogits=P + 16), "overlaps"), (dict(dlogits=P, grad_stride=1008), "overlaps"), (dict(dlogits=P + 1600, grad_stride=1500, row_stride=1500), "overlaps"),
    ],
    "iris_distill_topk": [
        (dict(list_k=129), "list_k"), (dict(list_k=-1), "list_k"), (dict(mode=2), "mode"), (dict(teacher=None), "teacher is NULL"), (dict(teacher_ids=None), "teacher_ids"),
        (dict(teacher_ids=P + 4), "teacher_ids"), (dict(teacher_scale=0.0), "teacher_scale"), (dict(loss=None), "loss is NULL"), (dict(weight=P + 1), "weight"),
        (dict(dlogits=P + 32), "overlaps"), (dict(dlogits=P - 32), "overlaps"), (dict(dlogits=P, grad_stride=900), "row stride"),
    ],
    "iris_distill_topk_backward": [
        (dict(stats=None), "stats is NULL"), (dict(grad_loss=None), "weight is NULL"), (dict(dlogits=None), "dlogits is NULL"), (dict(dlogits=P + 8), "overlaps"),
        (dict(list_k=200), "list_k"), (dict(mode=-1), "mode"),
    ],
}


@pytest.mark.parametrize("call,change,says", [(c, *x) for c in CALLS for x in COMMON + OWN[c]])
def test_refusals(call, change, says):
    with pytest.raises(iris.IrisError) as e:
        getattr(iris, call)(**{**CALLS[call], **change})
    assert e.value.code == iris.IRIS_ERR_ARG and says in str(e.value)


@pytest.mark.parametrize("call", sorted(CALLS))
def test_sizes_beyond_the_limits(call):
    for change in (dict(rows=1 << 31), dict(vocab=(1 << 30) + 1)):
        with pytest.raises(iris.IrisError) as e:
            getattr(iris, call)(**{**CALLS[call], **change})
        assert e.value.code == iris.IRIS_ERR_UNSUPPORTED


@pytest.mark.parametrize("call", sorted(CALLS))
def test_null_args_and_no_rows(call):
    assert getattr(iris.lib(), call)(None, None) == iris.IRIS_ERR_ARG
    none = {k: None for k, v in CALLS[call].items() if v == P}
    getattr(iris, call)(**{**CALLS[call], **none, "rows": 0, "dlogits": P} if "dlogits" in none else {**CALLS[call], **none, "rows": 0})


def test_the_matrix_product_keeps_to_16_bit_types():
    a = iris.GemmArgs()
    a.dtype = iris.IRIS_F32
    assert iris.lib().iris_gemm_all_scatter_ex(ctypes.byref(a), None) != iris.IRIS_OK
