"""Refusals of the optimizer's side that need no device."""
import ctypes

import pytest

from paper_2405_17517_b200 import binding as B
from paper_2405_17517_b200 import build as wash_build


@pytest.fixture(scope="module")
def lib():
    wash_build.build()
    return B.load()


def test_null_context(lib):
    norm = (ctypes.c_double * 4)()
    at = ctypes.addressof(norm)
    assert lib.wash_grad_norm(None, 0, 1, at, None) == B.WASH_ERR_ARG
    assert lib.wash_clip_grads(None, 1.0, at, None) == B.WASH_ERR_ARG
    assert lib.wash_set_decay(None, None, None) == B.WASH_ERR_ARG
    assert lib.wash_sgd_step(None, 0.1, 0.9, 0.0, 0, 1.0, at, None) == B.WASH_ERR_ARG
    assert lib.wash_adamw_step(None, 0, 0.1, 0.9, 0.999, 1e-8, 0.0, 0, 1.0, at, None) == B.WASH_ERR_ARG
    assert "ctx" in B.wash_last_error()


@pytest.mark.parametrize("args,word", [((0.1, 1.0, 0.0, 0), "momentum"), ((0.1, float("nan"), 0.0, 0), "momentum"), ((0.1, 0.9, 0.0, 8), "flags"),
                                       ((0.1, 0.0, 0.0, B.WASH_STEP_NESTEROV), "Nesterov")])
def test_sgd_arguments(lib, args, word):
    with pytest.raises(B.WashError) as e:
        B.wash_sgd_step(None, *args, stream=0)
    assert e.value.code == B.WASH_ERR_ARG and word in str(e.value)


@pytest.mark.parametrize("kw,word", [(dict(step=1 << 56), "step"), (dict(beta1=1.0), "beta1"), (dict(beta2=-0.1), "beta2"), (dict(eps=0.0), "eps"),
                                     (dict(eps=1e-50), "eps"), (dict(flags=B.WASH_STEP_NESTEROV), "flags")])
def test_adamw_arguments(lib, kw, word):
    with pytest.raises(B.WashError) as e:
        B.wash_adamw_step(None, kw.pop("step", 0), 0.1, stream=0, **kw)
    assert e.value.code == B.WASH_ERR_ARG and word in str(e.value)


def test_norms_are_float64_device_tensors(lib):
    import numpy as np
    import torch
    for norm in (torch.zeros(4, dtype=torch.float64), torch.zeros(4), np.zeros(4)):       # host memory would be read by the GPU
        for call in (lambda: B.wash_grad_norm(None, 0, 1, norm, stream=0), lambda: B.wash_clip_grads(None, 1.0, norm, stream=0),
                     lambda: B.wash_sgd_step(None, 0.1, max_norm=1.0, dev_norm=norm, stream=0), lambda: B.wash_adamw_step(None, 0, 0.1, max_norm=1.0, dev_norm=norm, stream=0)):
            with pytest.raises(TypeError):
                call()
