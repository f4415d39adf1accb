"""What the library reads and writes by a context's sizes -- N norms, a probability or a multiplier a tensor -- has to be there: arrays that are
too short, and norms on another device, are refused before the call.  The library is a stand-in that takes every call, so no device is needed."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2405_17517_b200 import binding as B


class Library:
    """Takes every call and keeps the names and the last arguments; contexts are numbered from 4096."""

    def __init__(self):
        self.calls, self.made, self.last = [], 0, ()

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            self.last = args
            if name in ("wash_create", "wash_create_segments"):
                self.made += 1
                args[0]._obj.value = 4096 * self.made
            return 0
        return call


class Norms:
    """What the binding asks of a CUDA tensor"""
    is_cuda = True

    def __init__(self, count, device, dtype=torch.float64):
        self.count, self.device, self.dtype = count, device, dtype

    def is_contiguous(self):
        return True

    def numel(self):
        return self.count

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def library(monkeypatch):
    lib, populations, start = Library(), [], B.Population.__init__

    def kept(self, *args, **kw):
        populations.append(self)
        start(self, *args, **kw)

    monkeypatch.setattr(B, "load", lambda: lib)
    monkeypatch.setattr(B.Population, "__init__", kept)
    yield lib
    for population in populations:      # a made-up handle must not reach the library itself
        population.close()


def _norm_calls(ctx, norm):
    return [lambda: B.wash_grad_norm(ctx, 0, 3, norm, stream=0), lambda: B.wash_clip_grads(ctx, 1.0, norm, stream=0),
            lambda: B.wash_sgd_step(ctx, 0.1, max_norm=1.0, dev_norm=norm, stream=0), lambda: B.wash_adamw_step(ctx, 0, 0.1, max_norm=1.0, dev_norm=norm, stream=0)]


@pytest.mark.parametrize("create", [lambda: B.wash_create(4, [5, 6, 7], 0, 1), lambda: B.wash_create_segments(4, [5, 6, 7], layout=1, device=1),
                                    lambda: B.Population(4, [5, 6, 7], 0, 1)], ids=["create", "segments", "population"])
def test_norms_are_n_doubles_on_the_contexts_device(library, create):
    made = create()                                                     # (a population closes its context when it is dropped)
    ctx = made if isinstance(made, int) else made.ctx
    for norm in (Norms(3, 1), Norms(0, 1), Norms(4, 0), Norms(64, 2)):
        before = list(library.calls)
        for call in _norm_calls(ctx, norm):
            with pytest.raises(ValueError):
                call()
        assert library.calls == before
    for norm in (Norms(4, 1), Norms(5, 1), 1 << 20):                    # an address is the caller's word
        before = len(library.calls)
        for call in _norm_calls(ctx, norm):
            call()
        assert len(library.calls) == before + 4
    with pytest.raises(TypeError):
        B.wash_grad_norm(ctx, 0, 3, Norms(4, 1, torch.float32), stream=0)


def _tensor_calls(ctx, values):
    return [lambda: B.wash_set_decay(ctx, values, stream=0), lambda: B.wash_shuffle(ctx, 0, 0.1, values, stream=0),
            lambda: B.wash_shuffle_opt_state(ctx, 0, 0.1, values, stream=0), lambda: B.wash_shuffle_both(ctx, 0, 0.1, values, stream=0),
            lambda: B.wash_shuffle_consensus(ctx, 0, 0, 0.1, values, stream=0, tensor_bounds=(0, 3), dev_sq_out=1 << 20),
            lambda: B.wash_step_host(ctx, B.WASH_OP_SHUFFLE, 1 << 20, None, None, 0, 0.1, values, stream=0), lambda: B.wash_exchange_plan(ctx, 0, 0.1, values, stream=0),
            lambda: B.wash_shuffle_noalloc(4, [5, 6, 7], 0, B.WASH_F32, 1 << 20, 96, 0, 0.1, values, stream=0)]


def test_arrays_have_a_value_for_every_tensor(library):
    ctx = B.wash_create(4, [5, 6, 7])
    for values in ([], [0.1, 0.2], np.zeros(2), 0.5):
        before = list(library.calls)
        for call in _tensor_calls(ctx, values):
            with pytest.raises(ValueError):
                call()
        assert library.calls == before
    for values in ([0.1, 0.2, 0.3], (0.0, 1.0, 0.5), np.zeros(3, np.float32), np.zeros(9), None):
        before = len(library.calls)
        for call in _tensor_calls(ctx, values):
            call()
        assert len(library.calls) == before + 8


def test_a_destroyed_contexts_sizes_are_forgotten(library):
    ctx = B.wash_create(64, [5] * 9)
    B.wash_destroy(ctx)
    B.wash_set_decay(ctx, [1.0], stream=0)                               # a handle that is not known is passed on as it is
    other = B.wash_create(2, [5])
    B.wash_set_decay(other, [1.0], stream=0)
    B.wash_grad_norm(other, 0, 1, Norms(2, 0), stream=0)


def test_norms_come_with_a_bound(library):
    """A step that is given norms and no bound would run with the bound 0, which takes all gradients away."""
    ctx = B.wash_create(4, [5, 6, 7])
    before = list(library.calls)
    for norm in (Norms(4, 0), 1 << 20):
        for call in (lambda: B.wash_sgd_step(ctx, 0.1, 0.9, dev_norm=norm, stream=0), lambda: B.wash_adamw_step(ctx, 0, 0.1, dev_norm=norm, stream=0),
                     lambda: B.wash_sgd_step(ctx, 0.1, flags=B.WASH_STEP_SKIP_NONFINITE, dev_norm=norm, stream=0)):
            with pytest.raises(ValueError):
                call()
    assert library.calls == before
    for bound in (0.0, 0, 2.5):                                          # 0 is what it says when it is asked for
        B.wash_sgd_step(ctx, 0.1, 0.9, 0.0, 0, bound, Norms(4, 0), stream=0)
        assert library.last[5] == bound and library.last[6] == 1 << 20
        B.wash_adamw_step(ctx, 0, 0.1, max_norm=bound, dev_norm=Norms(4, 0), stream=0)
        assert library.last[8] == bound and library.last[9] == 1 << 20
    for bound in (None, 0.0, 2.5):                                       # ignored without norms
        B.wash_sgd_step(ctx, 0.1, 0.9, max_norm=bound, stream=0)
        assert library.last[6] is None
        B.wash_adamw_step(ctx, 0, 0.1, max_norm=bound, stream=0)
        assert library.last[9] is None


def test_stacks_lie_on_the_populations_device(library):
    """The kernels run on the context's device; a stack of another one is memory that they may not reach."""
    pop = B.Population(4, [5, 6, 7], 0, 1)
    before = list(library.calls)
    for role in (B.WASH_STACK_PARAMS, B.WASH_STACK_OPT, B.WASH_STACK_GRADS, B.WASH_STACK_OPT2):
        for device in (0, 2):
            with pytest.raises(ValueError):
                pop.bind(role, Norms(96, device, torch.float32))
    assert library.calls == before
    for role in (B.WASH_STACK_PARAMS, B.WASH_STACK_OPT, B.WASH_STACK_GRADS, B.WASH_STACK_OPT2):
        pop.bind(role, Norms(96, 1, torch.float32))
    assert library.calls == before + ["wash_bind"] * 4
