"""Momentum and the betas are below 1 as the kernels hold them, in binary32: a weight that rounds to 1 would never forget, while new terms still come in.
No device is needed: these arguments are looked at before the context."""
import pytest

from paper_2405_17517_b200 import binding as B
from paper_2405_17517_b200 import build as wash_build

CLOSE = [1.0 - 2.0 ** -25, 1.0 - 1e-9, 1.0 - 2.0 ** -53]       # round to 1 in binary32; the first is a tie, which goes to the even 1


@pytest.fixture(scope="module", autouse=True)
def lib():
    wash_build.build()


def _refusal(call, *args, **kw):
    with pytest.raises(B.WashError) as e:
        call(None, *args, stream=0, **kw)
    assert e.value.code == B.WASH_ERR_ARG
    return str(e.value)


@pytest.mark.parametrize("weight", CLOSE)
def test_weights_that_round_to_one_are_refused(weight):
    assert "momentum" in _refusal(B.wash_sgd_step, 0.1, weight)
    assert "momentum" in _refusal(B.wash_sgd_step, 0.1, weight, 0.0, B.WASH_STEP_NESTEROV)
    assert "beta1" in _refusal(B.wash_adamw_step, 0, 0.1, beta1=weight)
    assert "beta2" in _refusal(B.wash_adamw_step, 0, 0.1, beta2=weight)


@pytest.mark.parametrize("weight", [1.0 - 2.0 ** -24, 1.0 - 2.0 ** -25 - 2.0 ** -50, 0.9999, 0.5, 0.0, 1e-60])
def test_weights_below_are_not(weight):
    """only the missing context is wrong with these"""
    for call, args, kw in ((B.wash_sgd_step, (0.1, weight), {}), (B.wash_adamw_step, (0, 0.1), dict(beta1=weight)), (B.wash_adamw_step, (0, 0.1), dict(beta2=weight))):
        assert "ctx" in _refusal(call, *args, **kw)
