"""What the operators around the head refuse, before anything is launched (no GPU needed): arguments, sizes, workspaces, tensors that are not what the call
takes them for."""
import numpy as np
import pytest
import torch

import paper_2511_12500_b200 as iris
from paper_2511_12500_b200 import binding, build as iris_build

P = 1 << 20   # an address that nothing reads: every call here is refused first


@pytest.fixture(scope="module", autouse=True)
def library():
    iris_build.build()


BF16 = iris.IRIS_BF16
VERIFY = dict(logits=P, sequences=3, drafts=2, vocab=1000, dtype=BF16, draft_ids=P, uniform=P, noise=P, tokens=P, accepted=P, workspace=P, draft_logits=P, logprob=P,
              scales=P, stream=0)
EMBED = dict(shards=[P, P], vocab=1000, dim=64, dtype=BF16, tokens=P, n=5, out=P, stream=0)
EMBED_GRAD = dict(grad_out=P, n=5, dim=64, dtype=BF16, tokens=P, grad_shards=[P, P], vocab=1000, grad_dtype=iris.IRIS_F32, workspace=P, stream=0)
NORM = dict(x=P, rows=4, dim=96, dtype=BF16, y=P, weight=P, bias=P, stats=P, stream=0)
NORM_GRAD = dict(x=P, rows=4, dim=96, dtype=BF16, dy=P, stats=P, workspace=P, weight=P, dx=P, dweight=P, dbias=P, stream=0)
CALLS = {"iris_verify_drafts": VERIFY, "iris_embed_tokens": EMBED, "iris_embed_tokens_backward": EMBED_GRAD, "iris_layer_norm": NORM,
         "iris_layer_norm_backward": NORM_GRAD}
INF, NAN = float("inf"), float("nan")
REFUSED = {
    "iris_verify_drafts": [
        (dict(dtype=3), "dtype"), (dict(sequences=-1), "sequences"), (dict(drafts=-1), "drafts"), (dict(drafts=129), "drafts"), (dict(vocab=0), "vocab"),
        (dict(vocab=-3), "vocab"), (dict(row_stride=999), "row stride"), (dict(draft_stride=999), "row stride"), (dict(logits=None), "logits is NULL"),
        (dict(logits=P + 1), "aligned"), (dict(draft_logits=P + 1), "aligned"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=NAN), "scale"),
        (dict(scales=P + 2), "scales"), (dict(draft_ids=None), "draft_ids is NULL"), (dict(draft_ids=P + 4), "draft_ids"), (dict(uniform=None), "uniform is NULL"),
        (dict(noise=None), "noise is NULL"), (dict(scale=INF, noise=None), "noise is NULL"), (dict(noise=P + 2), "noise"), (dict(tokens=None), "tokens is NULL"),
        (dict(tokens=P + 4), "tokens"), (dict(accepted=None), "accepted is NULL"), (dict(logprob=P + 1), "logprob"), (dict(workspace=None), "workspace is NULL"),
        (dict(workspace=P + 8), "workspace"), (dict(row_stride=1 << 61), "too large"),
    ],
    "iris_embed_tokens": [
        (dict(dtype=5), "dtype"), (dict(shards=[]), "world=0"), (dict(shards=[P] * 9), "world=9"), (dict(vocab=-2), "vocab"), (dict(vocab=1001), "multiple of world"),
        (dict(dim=-1), "dim"), (dict(n=-1), "n="), (dict(shard_stride=63), "row stride"), (dict(out_stride=63), "row stride"), (dict(shards=[P, P + 1]), "shard"),
        (dict(out=None), "out is NULL"), (dict(out=P + 1), "out"), (dict(tokens=None), "tokens is NULL"), (dict(tokens=P + 4), "tokens"), (dict(scale=INF), "scale"),
        (dict(scale=NAN), "scale"),
    ],
    "iris_embed_tokens_backward": [
        (dict(dtype=5), "dtype"), (dict(grad_dtype=iris.IRIS_F16), "grad_dtype"), (dict(grad_dtype=7), "grad_dtype"), (dict(grad_shards=[]), "world=0"),
        (dict(vocab=1001), "multiple of world"), (dict(n=-4), "n="), (dict(shard_stride=63), "row stride"), (dict(grad_out_stride=63), "row stride"),
        (dict(grad_out=None), "grad_out is NULL"), (dict(grad_shards=[P, P + 2]), "grad_shard"), (dict(tokens=None), "tokens is NULL"), (dict(scale=INF), "scale"),
        (dict(workspace=None), "workspace is NULL"), (dict(workspace=P + 4), "workspace"),
    ],
    "iris_layer_norm": [
        (dict(dtype=-1), "dtype"), (dict(param_dtype=iris.IRIS_F16), "param_dtype"), (dict(rows=-1), "rows"), (dict(dim=0), "dim"), (dict(row_stride=95), "row stride"),
        (dict(out_stride=95), "row stride"), (dict(x=None), "x is NULL"), (dict(x=P + 1), "x"), (dict(y=None), "y is NULL"), (dict(weight=P + 2), "weight"),
        (dict(bias=P + 2), "bias"), (dict(stats=P + 4), "stats"), (dict(eps=-1e-5), "eps"), (dict(eps=NAN), "eps"), (dict(eps=INF), "eps"), (dict(y=P + 16), "overlaps"),
        (dict(y=P, out_stride=104), "overlaps"),
    ],
    "iris_layer_norm_backward": [
        (dict(dtype=-1), "dtype"), (dict(param_dtype=iris.IRIS_F16), "param_dtype"), (dict(dim=0), "dim"), (dict(row_stride=95), "row stride"),
        (dict(dy_stride=95), "row stride"), (dict(dx_stride=95), "row stride"), (dict(dy=None), "dy is NULL"), (dict(stats=None), "stats is NULL"),
        (dict(dx=P + 32), "overlaps x"), (dict(dx=P + 4096, dy=P + 4096 - 32), "overlaps dy"), (dict(workspace=None), "workspace is NULL"), (dict(dweight=P + 2), "dweight"),
        (dict(dbias=P + 2), "dbias"), (dict(weight=P + 2), "weight"),
    ],
}


def refused(call, says, code=iris.IRIS_ERR_ARG, **change):
    with pytest.raises(iris.IrisError) as e:
        getattr(iris, call)(**{**CALLS[call], **change})
    assert e.value.code == code and says in str(e.value), str(e.value)


@pytest.mark.parametrize("call,change,says", [(c, *x) for c in CALLS for x in REFUSED[c]])
def test_refusals(call, change, says):
    refused(call, says, **change)


@pytest.mark.parametrize("call,change", [
    ("iris_verify_drafts", dict(vocab=(1 << 30) + 1)), ("iris_verify_drafts", dict(sequences=1 << 28)), ("iris_embed_tokens", dict(n=(1 << 30) + 1)),
    ("iris_embed_tokens", dict(vocab=1 << 31)), ("iris_embed_tokens", dict(dim=(1 << 24) + 1)), ("iris_embed_tokens_backward", dict(n=(1 << 30) + 1)),
    ("iris_embed_tokens_backward", dict(dim=(1 << 24) + 1)), ("iris_layer_norm", dict(dim=65537)), ("iris_layer_norm", dict(rows=1 << 31)),
    ("iris_layer_norm_backward", dict(dim=65537))])
def test_sizes_beyond_the_limits(call, change):
    refused(call, "", iris.IRIS_ERR_UNSUPPORTED, **change)


@pytest.mark.parametrize("call", sorted(CALLS))
def test_null_args(call):
    assert getattr(iris.lib(), call)(None, None) == iris.IRIS_ERR_ARG


def test_nothing_to_do():
    """No rows, sequences or tokens: nothing is looked at, nothing is launched."""
    iris.iris_verify_drafts(**{**{k: None if v == P else v for k, v in VERIFY.items()}, "sequences": 0})
    iris.iris_embed_tokens(**{**EMBED, "n": 0, "out": None, "tokens": None})
    iris.iris_embed_tokens_backward(**{**EMBED_GRAD, "grad_shards": [None, None], "workspace": None})
    iris.iris_embed_tokens_backward(**{**EMBED_GRAD, "n": 0, "accumulate": True, "workspace": None, "tokens": None, "grad_out": None})
    iris.iris_layer_norm(**{**NORM, "rows": 0, "x": None, "y": None})
    iris.iris_layer_norm_backward(**{**NORM_GRAD, "dx": None, "dweight": None, "dbias": None, "workspace": None})


def test_workspaces_that_are_too_small():
    """What a workspace holds is told by its tensor; here by the argument block itself."""
    for call, args in (("iris_verify_drafts", (P, 3, 1000, 0, 2, BF16, 1.0, 0, P, 0, P, P, P, P, P, P, P, iris.iris_verify_workspace_bytes(3, 2) - 1)),
                       ("iris_embed_tokens_backward", (P, 5, 64, 0, BF16, 2, P, P, P, 0, 0, 0, 0, 0, 0, 2, 0, 1000, 0, 1.0, P, iris.iris_embed_workspace_bytes(5, 1000, 64) - 1)),
                       ("iris_layer_norm_backward", (P, P + (1 << 16), 4, 96, 0, 0, BF16, 2, P, P, P + (1 << 17), 0, P, P, P, iris.iris_layer_norm_workspace_bytes(4, 96) - 1))):
        form = {"iris_verify_drafts": binding._VERIFY_ARGS, "iris_embed_tokens_backward": binding._EMBED_GRAD_ARGS,
                "iris_layer_norm_backward": binding._LAYER_NORM_GRAD_ARGS}[call]
        assert getattr(iris.lib(), call)(form.pack(*args), None) == iris.IRIS_ERR_ARG
        assert "workspace has" in iris.iris_last_error(), iris.iris_last_error()


def test_workspace_sizes():
    assert iris.iris_verify_workspace_bytes(0, 3) == iris.iris_verify_workspace_bytes(4, 129) == iris.iris_layer_norm_workspace_bytes(0, 5) == 0
    assert iris.iris_layer_norm_workspace_bytes(5, 65537) == iris.iris_embed_workspace_bytes(-1, 5, 5) == 0
    assert iris.iris_verify_workspace_bytes(2, 3) == 2 * iris.iris_verify_workspace_bytes(1, 3) > 0
    for rows, dim in ((1, 1), (10, 4096), (1 << 20, 64), (1 << 20, 65536)):
        assert iris.iris_layer_norm_workspace_bytes(rows, dim) >= 8 * dim
    for n, vocab, dim in ((0, 8, 8), (1, 8, 8), (1 << 20, 160000, 8192)):
        assert iris.iris_embed_workspace_bytes(n, vocab, dim) >= 16 * n + vocab // 8


# ------------------------------------------------------------------------------------------------- tensors
# name -> (type, rows, columns); rows None: a contiguous buffer of `columns` elements
B16, F32, I64, U8 = torch.bfloat16, torch.float32, torch.int64, torch.uint8
TENSORS = {
    "iris_verify_drafts": dict(logits=(B16, 9, 1000), draft_logits=(B16, 6, 1000), draft_ids=(I64, None, 6), uniform=(F32, None, 6), noise=(F32, None, 3000),
                               tokens=(I64, None, 9), accepted=(I64, None, 3), logprob=(F32, None, 9), scales=(F32, None, 3)),
    "iris_embed_tokens": dict(tokens=(I64, None, 5), out=(B16, 5, 64)),
    "iris_embed_tokens_backward": dict(tokens=(I64, None, 5), grad_out=(B16, 5, 64)),
    "iris_layer_norm": dict(x=(B16, 4, 96), y=(B16, 4, 96), weight=(F32, None, 96), bias=(F32, None, 96), stats=(F32, None, 8)),
    "iris_layer_norm_backward": dict(x=(B16, 4, 96), dy=(B16, 4, 96), dx=(B16, 4, 96), weight=(F32, None, 96), dweight=(F32, None, 96), dbias=(F32, None, 96),
                                     stats=(F32, None, 8)),
}
STRIDE = {"logits": "row_stride", "draft_logits": "draft_stride", "out": "out_stride", "grad_out": "grad_out_stride", "x": "row_stride", "y": "out_stride",
          "dy": "dy_stride", "dx": "dx_stride"}


@pytest.mark.parametrize("call,name", [(c, n) for c in TENSORS for n in TENSORS[c]])
def test_tensors_that_are_not_what_the_call_needs(call, name):
    dtype, rows, columns = TENSORS[call][name]
    size = (rows or 1) * columns
    for wrong in (torch.float64, torch.int32):
        refused(call, f"{name} is {wrong}, not {dtype}", **{name: torch.zeros(size, dtype=wrong)})
    refused(call, f"{name} is a ndarray", **{name: np.zeros(size)})
    if rows is None:
        refused(call, f"{name} is not contiguous", **{name: torch.zeros(1, dtype=dtype).expand(size)})
        refused(call, f"{name} has {size - 1} elements", **{name: torch.zeros(size - 1, dtype=dtype)})
        refused(call, f"{name} is not on the GPU", **{name: torch.zeros(size, dtype=dtype)})
        return
    stride = STRIDE[name]
    refused(call, "the row stride is not given", **{name: torch.zeros(rows, columns + 8, dtype=dtype)})
    refused(call, "elements apart", **{name: torch.zeros(columns, rows, dtype=dtype).t(), stride: columns})
    refused(call, "does not hold", **{name: torch.zeros(rows - 1, columns, dtype=dtype)})
    refused(call, "does not hold", **{name: torch.zeros(rows, columns, dtype=dtype), stride: columns + 1})
    refused(call, "does not hold", **{name: torch.zeros(1, columns, dtype=dtype).expand(rows, columns), stride: columns})
    refused(call, f"{name} is not on the GPU", **{name: torch.zeros(rows, columns, dtype=dtype)})
    refused(call, f"{name} is not on the GPU", **{name: torch.zeros(rows, columns + 8, dtype=dtype)[:, 3:columns + 3], stride: columns + 8})


@pytest.mark.parametrize("call,name", [("iris_embed_tokens", "shards"), ("iris_embed_tokens_backward", "grad_shards")])
def test_shards_that_are_not_what_the_call_needs(call, name):
    dtype = B16 if name == "shards" else F32
    good = torch.zeros(500, 64, dtype=dtype)
    for bad, says in ((torch.zeros(500, 64, dtype=torch.float64), "not torch"), (good[:499], "does not hold"), (torch.zeros(64, 500, dtype=dtype).t(), "row stride is not"),
                      (good, "not on the GPU")):
        with pytest.raises(iris.IrisError) as e:
            getattr(iris, call)(**{**CALLS[call], name: [P, bad]})
        assert e.value.code == iris.IRIS_ERR_ARG and name[:-1] in str(e.value) and (says in str(e.value) or "elements apart" in str(e.value)), str(e.value)


def test_the_extension_takes_what_is_right():
    binding._first_call()
    assert binding._accept_rows.__self__.__name__ == "paper_2511_12500_b200._tensors"
    take = binding._accept_rows
    assert take(0, P, 1, 3, 50, 0, None, 2, 3, 50, 0) == (P, 0)
    assert take(0, torch.zeros(3, 50), 2, 0, 50, 0) is None   # on the CPU
    for bad in ((), (0, P, 1, 3), ("a", P, 1, 3, 50, 0), (0, "x", 1, 3, 50, 0), (0, torch.zeros(3, 50), "y", 3, 50, 0), (0, -1, 1, 3, 50, 0)):
        assert take(*bad) is None
