"""More of what the operators on logits refuse before anything is launched (no GPU needed): scales whose exponents overflow."""
import pytest

import paper_2511_12500_b200 as iris
from paper_2511_12500_b200 import build as iris_build
from test_logit_ops_args import CALLS


@pytest.fixture(scope="module", autouse=True)
def library():
    iris_build.build()


@pytest.mark.parametrize("call", sorted(CALLS))
def test_scales_whose_exponents_overflow(call):
    with pytest.raises(iris.IrisError) as e:
        getattr(iris, call)(**{**CALLS[call], "scale": 2.5e38})
    assert e.value.code == iris.IRIS_ERR_ARG and "scale is at most 2e+38" in str(e.value)
