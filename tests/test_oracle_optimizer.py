"""Pins of the oracle's optimizer side: binary64 restatements on dense arrays, with bounds derived from the number of roundings."""
import numpy as np
import pytest

import oracle
import optimizer_reference as R
from paper_2405_17517_b200 import workloads as W

NUMEL = [37, 8, 1, 130, 5]
DECAY = [1.0, 0.0, 0.5, 1.0, 0.0]


def _case(N, layout, seed, wdtype="f32", gdtype="f32"):
    off, P = W.padded_offsets(NUMEL)
    pop = oracle.Population(N, NUMEL, off, P, layout)
    total = sum(NUMEL)
    out = []
    for k, (dtype, std) in enumerate(((wdtype, 0.05), (gdtype, 0.3), ("f32", 0.1), ("f32", 0.2))):
        dense = W.flat_population(N, total, seed=seed + k, std=std)
        if k == 3:
            dense = dense * dense
        bits = W.to_bf16_bits(dense) if dtype == "bf16" else dense
        out.append((W.bf16_bits_to_f32(bits) if dtype == "bf16" else dense, W.to_stack(bits, NUMEL, off, P, layout)))
    return pop, off, P, out


def _dense(stack, N, off, P, layout):
    d = W.from_stack(stack, N, NUMEL, off, P, layout)
    return W.bf16_bits_to_f32(d) if d.dtype == np.uint16 else d


def _wd(weight_decay):
    return weight_decay * np.repeat(DECAY, NUMEL)


def _padding_untouched(stack, off, P, N, layout):
    row = stack.reshape(N, P) if layout == 0 else stack.reshape(P, N).T
    pad = np.ones(P, bool)
    for d, o in zip(NUMEL, off):
        pad[o:o + d] = False
    vals = row[:, pad]
    return (vals == 0xFFFF).all() if vals.dtype == np.uint16 else np.isnan(vals).all()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_and_clip(dtype, layout):
    N = 5
    pop, off, P, st = _case(N, layout, 3, gdtype=dtype)
    dense, stack = st[1]
    want = np.sqrt((dense.astype(np.float64) ** 2).sum(1))
    norm = oracle.grad_norm(pop, stack)
    # 181 squares, added one after the other in binary64
    assert np.allclose(norm, want, rtol=200 * 2.0 ** -53, atol=0)
    lo, hi = 1, 4
    part = dense[:, NUMEL[0]:sum(NUMEL[:hi])].astype(np.float64)
    assert np.allclose(oracle.grad_norm(pop, stack, lo, hi), np.sqrt((part ** 2).sum(1)), rtol=200 * 2.0 ** -53, atol=0)
    assert (oracle.grad_norm(pop, stack, 2, 2) == 0).all()
    max_norm = float(np.sort(norm)[2])           # two models above, two below, one at the border (its factor is just below 1)
    before = stack.copy()
    oracle.clip_grads(pop, stack, max_norm, norm)
    c = R.factor(norm, max_norm)
    got = _dense(stack, N, off, P, layout)
    exact = dense * c[:, None]
    bound = 2.0 ** -23 * np.abs(exact)            # the factor and the product
    assert (np.abs(got - exact) <= bound + R.rounding(np.abs(exact) + bound, dtype == "bf16")).all()
    old = _dense(before, N, off, P, layout)
    for n in range(N):
        if np.float32(c[n]) == 1:
            assert (got[n] == old[n]).all()
        elif c[n] < 1 - 2.0 ** -7:                # more than the largest rounding (the model at the border may round back to itself in bf16)
            assert (got[n] != old[n]).all()
    assert _padding_untouched(stack, off, P, N, layout)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("wdtype,gdtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("momentum,nesterov", [(0.0, False), (0.9, False), (0.9, True)])
def test_sgd(momentum, nesterov, wdtype, gdtype, layout):
    N = 4
    pop, off, P, st = _case(N, layout, 11, wdtype, gdtype)
    (p, ps), (g, gs), (m, ms), _ = st
    norm = np.array([0.5, 1.0, 3.0, 40.0])
    oracle.sgd_step(pop, ps, gs, ms, 0.1, momentum, 0.02, DECAY, nesterov, False, 1.5, norm)
    want_p, want_m, bp, bm = R.sgd(p, g, m, 0.1, momentum, _wd(0.02), R.factor(norm, 1.5), nesterov, wdtype == "bf16")
    assert (np.abs(_dense(ps, N, off, P, layout) - want_p) <= bp).all()
    if momentum:
        assert (np.abs(_dense(ms, N, off, P, layout) - want_m) <= bm).all()
    else:
        assert (_dense(ms, N, off, P, layout) == m).all()
    assert _padding_untouched(ps, off, P, N, layout)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("wdtype,gdtype", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("step", [0, 1, 1000, 10 ** 7])
def test_adamw(step, wdtype, gdtype, layout):
    N = 4
    pop, off, P, st = _case(N, layout, 21, wdtype, gdtype)
    (p, ps), (g, gs), (m, ms), (v, vs) = st
    norm = np.array([0.5, 1.0, 3.0, 40.0])
    oracle.adamw_step(pop, step, ps, gs, ms, vs, 0.01, 0.9, 0.995, 1e-6, 0.1, DECAY, False, 1.5, norm)
    want_p, want_m, want_v, bp, bm, bv = R.adamw(p, g, m, v, step, 0.01, 0.9, 0.995, 1e-6, _wd(0.1), R.factor(norm, 1.5), wdtype == "bf16")
    for stack, want, bound in ((ps, want_p, bp), (ms, want_m, bm), (vs, want_v, bv)):
        assert (np.abs(_dense(stack, N, off, P, layout) - want) <= bound).all()
        assert _padding_untouched(stack, off, P, N, layout)


def test_without_norms_nothing_is_clipped_and_skipped_models_keep_everything():
    N = 3
    pop, off, P, st = _case(N, 0, 31)
    (p, ps), (g, gs), (m, ms), (v, vs) = st
    one = ps.copy(), ms.copy(), vs.copy()
    oracle.adamw_step(pop, 4, ps, gs, ms, vs, 0.01, norm=None)
    oracle.adamw_step(pop, 4, one[0], gs, one[1], one[2], 0.01, max_norm=1.0, norm=[0.1, 0.2, 0.3])
    assert all((a.view(np.uint32) == b.view(np.uint32)).all() for a, b in zip(one, (ps, ms, vs)))
    before = [a.copy() for a in (ps, ms)]
    oracle.sgd_step(pop, ps, gs, ms, 0.1, 0.9, 0.0, None, False, True, 1.0, [np.inf, 0.5, np.nan])
    for now, old in zip((ps, ms), before):
        same = (now.view(np.uint32) == old.view(np.uint32)).reshape(N, P).all(1)
        assert same.tolist() == [True, False, True]
    oracle.sgd_step(pop, ps, gs, ms, 0.1, 0.9, 0.0, None, False, False, 1.0, [0.5, 0.5, np.nan])
    assert np.isnan(_dense(ps, N, off, P, 0)[2]).all() and np.isfinite(_dense(ps, N, off, P, 0)[:2]).all()


def test_momentum_from_zero_is_the_gradient_and_adam_starts_with_its_sign():
    """Closed forms of the first step: m = d; AdamW's ratio is g / (|g| + eps sqrt(1 - beta2))-like, 1 in size for gradients far above eps."""
    N = 2
    pop, off, P, st = _case(N, 0, 41)
    (p, ps), (g, gs), (m, ms), (v, vs) = st
    zero = np.zeros_like(ms)
    oracle.sgd_step(pop, ps, gs, zero, 0.1, 0.9)
    assert (_dense(zero, N, off, P, 0) == g).all()
    m0, v0, p0 = np.zeros_like(ms), np.zeros_like(ms), np.zeros_like(ms)
    big = np.abs(g) > 1e-3
    oracle.adamw_step(pop, 0, p0, gs, m0, v0, 1.0, 0.9, 0.999, 1e-12)
    assert np.allclose(_dense(p0, N, off, P, 0)[big], -np.sign(g)[big], rtol=20 * R.U + 1e-8, atol=0)
