"""The optimizer's side of a training step on the GPU: gradient norms, clipping, SGD and AdamW.  Steps and clipping use the oracle's
operations in its order, so they are bit-identical to it; against the binary64 statements (optimizer_reference.py) the bounds
count roundings.  Padding is NaN in every stack, so a read or write of it shows."""
import numpy as np
import pytest
import torch

import oracle
import optimizer_reference as R
from paper_2405_17517_b200 import binding as B
from paper_2405_17517_b200 import sharding
from paper_2405_17517_b200 import workloads as W
from gpu_util import bits, to_device, to_host_bits

pytestmark = pytest.mark.gpu

RAGGED = [1000, 33, 7, 1, 4, 8, 5003, 2048]
ODD = [(i * 37) % 61 + 1 for i in range(120)]        # many tensors to a tile, most with padding
ROLES = {"p": B.WASH_STACK_PARAMS, "g": B.WASH_STACK_GRADS, "m": B.WASH_STACK_OPT, "v": B.WASH_STACK_OPT2}


class Training:
    """A population with gradients and optimizer state on both sides."""

    def __init__(self, N, numel, layout=0, wdtype="f32", gdtype="f32", seed=0, decay=None, roles="pgmv", tensor_id=None, coord_begin=None, dense=None, device_offset=0):
        self.N, self.numel, self.layout = N, [int(d) for d in numel], layout
        self.gpu = B.Population(N, self.numel, layout, 0, tensor_id, coord_begin)
        self.P, self.off = self.gpu.padded_P, self.gpu.offsets
        self.ora = oracle.Population(N, self.numel, self.off, self.P, layout, tensor_id, coord_begin)
        self.decay = decay
        self.dense, self.host, self.dev = {}, {}, {}
        for k, (role, std) in enumerate((("p", 0.05), ("g", 0.02), ("m", 0.01), ("v", 0.02))):
            if role not in roles:
                continue
            d = dense[role] if dense else W.flat_population(N, sum(self.numel), seed=seed + 100 * k, std=std)
            if role == "v" and not dense:
                d = d * d
            if role == "g" and not dense:
                d = d * np.exp(np.linspace(-1.5, 1.5, N)).astype(np.float32)[:, None]    # norms below and above the bound
            dtype = {"p": wdtype, "g": gdtype}.get(role, "f32")
            value = W.to_bf16_bits(d) if dtype == "bf16" else d
            self.dense[role] = W.bf16_bits_to_f32(value) if dtype == "bf16" else d
            self.host[role] = W.to_stack(value, self.numel, self.off, self.P, layout)
            t = to_device(self.host[role])
            if device_offset:      # a stack that is 16-byte and no better aligned
                wide = torch.empty(t.numel() + device_offset, dtype=t.dtype, device="cuda")
                wide[device_offset:].copy_(t)
                t = wide[device_offset:]
            self.dev[role] = t
            self.gpu.bind(ROLES[role], self.dev[role])
        if decay is not None:
            B.wash_set_decay(self.gpu.ctx, decay)
        self.norm = torch.full((N,), float("nan"), dtype=torch.float64, device="cuda")

    def norms(self, lo=0, hi=None):
        B.wash_grad_norm(self.gpu.ctx, lo, len(self.numel) if hi is None else hi, self.norm)
        return self.norm.cpu().numpy()

    def assert_equal(self, roles="pgmv"):
        torch.cuda.synchronize()
        B.wash_check(self.gpu.ctx)
        for role in roles:
            if role in self.host:
                bad = np.flatnonzero(~same_bits(to_host_bits(self.dev[role]), bits(self.host[role])))
                assert bad.size == 0, "%s: %d elements differ, first at %d" % (role, bad.size, bad[0])

    def dense_of(self, role):
        b = to_host_bits(self.dev[role])
        b = b if b.dtype == np.uint16 else b.view(np.float32)
        d = W.from_stack(b, self.N, self.numel, self.off, self.P, self.layout)
        return W.bf16_bits_to_f32(d) if d.dtype == np.uint16 else d

    def close(self):
        self.gpu.close()


def same_bits(a, b):
    """equal bits, or NaN on both sides (an operation's NaN has no fixed payload)"""
    wide = (lambda x: (x.astype(np.uint32) << 16)) if a.dtype == np.uint16 else (lambda x: x)
    nan = lambda x: (wide(x) & 0x7FFFFFFF) > 0x7F800000
    return (a == b) | (nan(a) & nan(b))


def _decay(n):
    return [(1.0, 0.0, 0.5)[i % 3] for i in range(n)]


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [2, 3, 5, 7, 8, 16, 31, 33, 37, 64])
def test_norms(N, dtype, layout):
    for numel in (RAGGED, ODD, [1], [2048], [70001, 3]):
        c = Training(N, numel, layout, gdtype=dtype, seed=N, roles="g")
        # binary64 squares are exact; every sum is of non-negative terms, so n additions in any order are off by at most n 2^-53
        rtol = (sum(numel) + 4) * 2.0 ** -53
        want = np.sqrt((c.dense["g"].astype(np.float64) ** 2).sum(1))
        assert np.allclose(c.norms(), want, rtol=rtol, atol=0)
        first = c.norm.clone()
        c.norms()
        assert (first.view(torch.int64) == c.norm.view(torch.int64)).all()          # the order of the additions is fixed
        T = len(numel)
        for lo, hi in ((0, 1), (T // 2, T), (T - 1, T), (1, T - 1), (T // 3, T // 3)):
            if lo <= hi:
                assert np.allclose(c.norms(lo, hi), oracle.grad_norm(c.ora, c.host["g"], lo, hi), rtol=2 * rtol, atol=0)
        c.assert_equal("g")
        c.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_norms_of_many_blocks(layout):
    """More chunks than blocks, so that every block walks several; the last tensor ends inside an octet."""
    for N, dtype in ((2, "f32"), (5, "bf16"), (24, "f32")):
        c = Training(N, [3_000_001, 17, 999_999], layout, gdtype=dtype, seed=N, roles="g")
        want = np.sqrt((c.dense["g"].astype(np.float64) ** 2).sum(1))
        assert np.allclose(c.norms(), want, rtol=4e6 * 2.0 ** -53, atol=0)
        c.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_norms_of_extreme_values(layout):
    N, d = 6, 301
    g = np.full((N, d), 0.0, np.float32)
    g[0] = 3e38                       # squares beyond binary32
    g[1] = 1e-45                      # and below it
    g[2, 5] = np.inf
    g[3, 300] = np.nan
    g[4, 7], g[4, 8] = -np.inf, np.nan
    c = Training(N, [d], layout, roles="g", dense={"g": g})
    got = c.norms()
    want = np.sqrt((g.astype(np.float64) ** 2).sum(1))
    assert np.allclose(got[:2], want[:2], rtol=400 * 2.0 ** -53, atol=0) and got[1] > 0
    assert got[2] == np.inf and np.isnan(got[3]) and np.isnan(got[4]) and got[5] == 0
    c.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [2, 3, 5, 8, 15, 32, 37, 64])
def test_clipping(N, dtype, layout):
    for numel in (RAGGED, ODD, [1], [6000]):
        c = Training(N, numel, layout, gdtype=dtype, seed=N, roles="g")
        norm = c.norms()
        for max_norm in (float(np.median(norm)), 1e9, 0.37 * float(norm.min())):
            old = c.dense_of("g")
            B.wash_clip_grads(c.gpu.ctx, max_norm, c.norm)
            oracle.clip_grads(c.ora, c.host["g"], max_norm, norm)
            c.assert_equal("g")
            exact = old.astype(np.float64) * R.factor(norm, max_norm)[:, None]
            bound = 3 * R.U * np.abs(exact) + 2.0 ** -149      # the factor and the product
            assert (np.abs(c.dense_of("g") - exact) <= bound + R.rounding(np.abs(exact) + bound, dtype == "bf16")).all()
        c.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_clipping_leaves_unclipped_models_bits_alone(dtype, layout):
    """Signalling NaNs and negative zeros of models within the bound stay; NaN and infinite norms do what the formula says."""
    N, d = 6, 2500
    c = Training(N, [d, 3], layout, gdtype=dtype, roles="g")
    flat = c.dev["g"].view(torch.int32 if dtype == "f32" else torch.int16)
    rows = flat.view(N, c.P) if layout == 0 else flat.view(c.P, N).t()
    rows[1, 100:108] = 0x7F800001 if dtype == "f32" else 0x7F81            # a signalling NaN
    rows[1, 200] = -(1 << 31) if dtype == "f32" else -(1 << 15)            # -0
    before = flat.clone()
    c.norm.copy_(torch.tensor([0.5, 0.9, 4.0, float("inf"), float("nan"), 0.0], dtype=torch.float64))
    B.wash_clip_grads(c.gpu.ctx, 1.0, c.norm)
    now = c.dense_of("g")
    kept = (flat == before).view(N, c.P) if layout == 0 else (flat == before).view(c.P, N).t()
    assert kept[[0, 1, 5]].all()
    assert not kept[2, :d].all() and (now[3] == 0).all() and np.isnan(now[4]).all()
    c.norm.fill_(2.0)
    B.wash_clip_grads(c.gpu.ctx, 0.0, c.norm)                                # bound 0: all gradients vanish
    assert (c.dense_of("g")[[0, 2, 3, 5]] == 0).all()
    B.wash_check(c.gpu.ctx)
    c.close()


RULES = [("sgd", 0.0, False), ("sgd", 0.9, False), ("sgd", 0.9, True), ("adamw", 0.9, False)]


def _step(c, rule, momentum, nesterov, step, max_norm, norm, skip=False, lr=0.05, wd=0.02):
    flags = (B.WASH_STEP_NESTEROV if nesterov else 0) | (B.WASH_STEP_SKIP_NONFINITE if skip else 0)
    given = c.norm if norm is not None else None
    if rule == "sgd":
        B.wash_sgd_step(c.gpu.ctx, lr, momentum, wd, flags, max_norm, given)
        oracle.sgd_step(c.ora, c.host["p"], c.host["g"], c.host.get("m"), lr, momentum, wd, c.decay, nesterov, skip, max_norm, norm)
    else:
        B.wash_adamw_step(c.gpu.ctx, step, lr, momentum, 0.995, 1e-6, wd, flags, max_norm, given)
        oracle.adamw_step(c.ora, step, c.host["p"], c.host["g"], c.host["m"], c.host["v"], lr, momentum, 0.995, 1e-6, wd, c.decay, skip, max_norm, norm)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("wdtype,gdtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rule,momentum,nesterov", RULES)
@pytest.mark.parametrize("N", [2, 3, 5, 8, 21, 64])
def test_steps(N, rule, momentum, nesterov, wdtype, gdtype, layout):
    for numel in (RAGGED, ODD, [1], [6000]):
        c = Training(N, numel, layout, wdtype, gdtype, seed=N, decay=_decay(len(numel)))
        norm = c.norms().copy()
        max_norm = float(np.median(norm))
        wd = 0.02 * np.repeat(_decay(len(numel)), numel)
        for step in (0, 1, 700):
            old = {k: c.dense_of(k) for k in "pgmv"}
            clipped = step != 1                     # one of the steps without clipping
            _step(c, rule, momentum, nesterov, step, max_norm, norm if clipped else None)
            c.assert_equal()
            f = R.factor(norm, max_norm) if clipped else np.ones(N)
            if rule == "sgd":
                p, m, bp, bm = R.sgd(old["p"], old["g"], old["m"], 0.05, momentum, wd, f, nesterov, wdtype == "bf16")
                v = None
            else:
                p, m, v, bp, bm, bv = R.adamw(old["p"], old["g"], old["m"], old["v"], step, 0.05, momentum, 0.995, 1e-6, wd, f, wdtype == "bf16")
                assert (np.abs(c.dense_of("v") - v) <= bv).all()
            assert (np.abs(c.dense_of("p") - p) <= bp).all()
            if momentum:
                assert (np.abs(c.dense_of("m") - m) <= bm).all()
        c.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rule,momentum,nesterov", RULES)
def test_models_with_infinite_or_nan_norms_keep_everything(rule, momentum, nesterov, layout):
    for N, wdtype in ((5, "f32"), (24, "bf16")):
        c = Training(N, RAGGED, layout, wdtype, wdtype, seed=2)
        g = c.host["g"].reshape(N, c.P) if layout == 0 else c.host["g"].reshape(c.P, N).T
        g[1, 17] = np.inf if wdtype == "f32" else 0x7F80
        g[3, 2000] = np.nan if wdtype == "f32" else 0x7FC0
        c.dev["g"].copy_(to_device(c.host["g"]))
        norm = c.norms().copy()
        assert np.isinf(norm[1]) and np.isnan(norm[3])
        old = {k: to_host_bits(c.dev[k]).copy() for k in "pmv"}
        _step(c, rule, momentum, nesterov, 3, 1.0, norm, skip=True)
        c.assert_equal()
        for k in "pmv":
            now, was = (x.reshape(N, c.P) if layout == 0 else x.reshape(c.P, N).T for x in (to_host_bits(c.dev[k]), old[k]))
            assert (now[[1, 3]] == was[[1, 3]]).all()
        assert np.isfinite(c.dense_of("p")).all()
        _step(c, rule, momentum, nesterov, 3, 1.0, norm, skip=False)       # without the flag the NaN goes through
        c.assert_equal()
        assert np.isnan(c.dense_of("p")[3]).all()
        c.close()


@pytest.mark.parametrize("rule,momentum,nesterov", RULES)
def test_special_values_follow_the_oracle(rule, momentum, nesterov):
    N = 4
    dense = {"p": W.flat_population(N, 4000, 1), "g": W.flat_population(N, 4000, 2), "m": W.flat_population(N, 4000, 3), "v": W.flat_population(N, 4000, 4) ** 2}
    dense["g"][0, :8] = [np.inf, -np.inf, np.nan, 3e38, -3e38, 1e-45, -1e-45, 0]
    dense["g"][1] = 0
    dense["v"][1] = 0                                      # sqrt(0) + eps below m
    dense["v"][2] = np.float32(1e-40)
    dense["m"][2] = np.float32(1e-42)
    dense["p"][3, :4] = [np.inf, -0.0, 1e-45, 3.4e38]
    for layout in (0, 1):
        for wdtype in ("f32", "bf16"):
            c = Training(N, [3999, 1], layout, wdtype, "f32", dense={k: v.copy() for k, v in dense.items()})
            _step(c, rule, momentum, nesterov, 0, 0.0, None)
            c.assert_equal()
            c.close()


def test_plain_sgd_needs_no_state_and_touches_none():
    c = Training(3, RAGGED, 0, roles="pgm")
    c.gpu.bind(B.WASH_STACK_OPT, c.dev["m"])
    before = c.dev["m"].clone()
    B.wash_sgd_step(c.gpu.ctx, 0.1)
    assert (c.dev["m"].view(torch.int32) == before.view(torch.int32)).all()
    B.wash_bind(c.gpu.ctx, B.WASH_STACK_OPT, B.WASH_F32, None, 0)
    B.wash_sgd_step(c.gpu.ctx, 0.1)
    for _ in range(2):
        oracle.sgd_step(c.ora, c.host["p"], c.host["g"], None, 0.1)
    c.assert_equal("pg")
    c.close()


def test_stacks_that_are_only_16_byte_aligned():
    for layout in (0, 1):
        for dtype, shift in (("f32", 4), ("bf16", 8)):
            c = Training(5, RAGGED, layout, dtype, dtype, device_offset=8 if dtype == "bf16" else 4)
            assert c.dev["g"].data_ptr() % 32 == 16
            norm = c.norms().copy()
            assert np.allclose(norm, oracle.grad_norm(c.ora, c.host["g"]), rtol=1e-12, atol=0)
            B.wash_clip_grads(c.gpu.ctx, float(np.median(norm)), c.norm)
            oracle.clip_grads(c.ora, c.host["g"], float(np.median(norm)), norm)
            _step(c, "adamw", 0.9, False, 2, 1.0, norm)
            _step(c, "sgd", 0.9, True, 2, 1.0, norm)
            c.assert_equal()
            c.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rule,momentum,nesterov", RULES[1:])
def test_a_training_loop_with_shuffles(rule, momentum, nesterov, layout):
    """norm -> step with clipping -> shuffle of weights and momentum, several steps with new gradients, against the oracle."""
    N = 5
    c = Training(N, RAGGED, layout, seed=6, decay=_decay(len(RAGGED)))
    p_layer = B.wash_layer_probs(len(RAGGED), 0.3)
    for step in range(4):
        g = W.to_stack(W.flat_population(N, sum(RAGGED), seed=900 + step, std=0.02 * (step + 1)), c.numel, c.off, c.P, layout)
        c.host["g"][...] = g
        c.dev["g"].copy_(to_device(g))
        norm = c.norms().copy()
        assert np.allclose(norm, oracle.grad_norm(c.ora, c.host["g"]), rtol=1e-12, atol=0)
        _step(c, rule, momentum, nesterov, step, 3.0, norm)
        B.wash_shuffle_both(c.gpu.ctx, step, 0.0, p_layer, seed=5)
        oracle.shuffle(c.ora, c.host["p"], p_layer, seed=5, step=step, stack2=c.host["m"])
        B.papa_ema(c.gpu.ctx, B.WASH_STACK_PARAMS, 0.99)
        oracle.papa_ema(c.ora, c.host["p"], 0.99)
        c.assert_equal()
    c.close()


def test_shards_give_the_whole_populations_step():
    """Three shards of one population (as on three GPUs): squared norms add up, and the steps of the parts are the step of the whole."""
    N, numel = 4, [4001, 64, 7, 1200, 3, 36, 2048]
    whole = Training(N, numel, 0, seed=8)
    total = whole.norms().copy()
    parts, squares = [], torch.zeros(N, dtype=torch.float64, device="cuda")
    for segs in sharding.plan_shards(numel, 3):
        sizes, tid, begin = sharding.segment_arrays(segs)
        dense = {k: np.ascontiguousarray(np.concatenate([whole.dense[k][:, s] for s in sharding.dense_slices(numel, segs)], axis=1)) for k in "pgmv"}
        part = Training(N, sizes, 0, dense=dense, tensor_id=tid, coord_begin=begin)
        part.norms()
        squares += part.norm ** 2
        parts.append((segs, part))
    norm = squares.sqrt()
    assert np.allclose(norm.cpu().numpy(), total, rtol=1e-13, atol=0)
    bound = float(np.median(total))
    B.wash_adamw_step(whole.gpu.ctx, 3, 0.01, max_norm=bound, dev_norm=norm)
    for segs, part in parts:
        B.wash_adamw_step(part.gpu.ctx, 3, 0.01, max_norm=bound, dev_norm=norm)
        for k in "pmv":
            want = np.concatenate([whole.dense_of(k)[:, s] for s in sharding.dense_slices(numel, segs)], axis=1)
            assert (part.dense_of(k).view(np.uint32) == want.view(np.uint32)).all()
        part.close()
    whole.close()


@pytest.mark.parametrize("N,layout,wdtype", [(6, 0, "f32"), (6, 1, "f32"), (24, 1, "bf16"), (64, 0, "bf16")])
def test_a_captured_step_is_replayed(N, layout, wdtype):
    """Norm, step and clipping in one graph on a stream of their own: replays continue from the state they find and read the norms anew; an
    eager call of the same context between replays disturbs neither."""
    c = Training(N, [50001, 33], layout, wdtype, wdtype, seed=4, decay=[1.0, 0.0])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        B.wash_grad_norm(c.gpu.ctx, 0, 2, c.norm)
        B.wash_adamw_step(c.gpu.ctx, 0, 0.01, max_norm=2.0, dev_norm=c.norm)
        B.wash_clip_grads(c.gpu.ctx, 2.0, c.norm)
        with pytest.raises(B.WashError) as e:
            B.wash_set_decay(c.gpu.ctx, [0.5, 0.5])
        assert e.value.code == B.WASH_ERR_STATE
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        norm = oracle.grad_norm(c.ora, c.host["g"])
        assert np.allclose(c.norm.cpu().numpy(), norm, rtol=1e-12, atol=0)
        norm = c.norm.cpu().numpy()
        oracle.adamw_step(c.ora, 0, c.host["p"], c.host["g"], c.host["m"], c.host["v"], 0.01, weight_decay=0.01, decay=c.decay, max_norm=2.0, norm=norm)
        oracle.clip_grads(c.ora, c.host["g"], 2.0, norm)
        c.assert_equal()
        assert np.allclose(c.norms(1, 2), oracle.grad_norm(c.ora, c.host["g"], 1, 2), rtol=1e-12, atol=0)
    c.close()


def test_a_context_can_be_captured_from_its_first_call_on():
    c = Training(3, [777], 0, seed=4)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.wash_grad_norm(c.gpu.ctx, 0, 1, c.norm)
        B.wash_sgd_step(c.gpu.ctx, 0.1, 0.9, 0.01, max_norm=0.5, dev_norm=c.norm)
    graph.replay()
    torch.cuda.synchronize()
    oracle.sgd_step(c.ora, c.host["p"], c.host["g"], c.host["m"], 0.1, 0.9, 0.01, max_norm=0.5, norm=c.norm.cpu().numpy())
    c.assert_equal()
    c.close()


def test_decay_multipliers_are_state_and_shuffles_keep_them():
    c = Training(3, RAGGED, 0, seed=9)
    for decay, p in ((None, 0.2), (_decay(len(RAGGED)), 0.2), (_decay(len(RAGGED)), 0.7), (None, 0.7)):
        B.wash_set_decay(c.gpu.ctx, decay)
        c.decay = decay
        B.wash_shuffle(c.gpu.ctx, 1, p, None, seed=3)        # uploads the table when p changes
        oracle.shuffle(c.ora, c.host["p"], p, seed=3, step=1)
        _step(c, "sgd", 0.9, False, 0, 0.0, None)
        c.assert_equal()
    bad = _decay(len(RAGGED))
    for value in (-1.0, float("nan"), float("inf"), 1e39):
        bad[3] = value
        with pytest.raises(B.WashError) as e:
            B.wash_set_decay(c.gpu.ctx, bad)
        assert e.value.code == B.WASH_ERR_ARG
    _step(c, "sgd", 0.9, False, 0, 0.0, None)                # the refused multipliers changed nothing
    c.assert_equal()
    c.close()


def test_calls_on_two_contexts_and_streams_do_not_disturb_each_other():
    cases = [Training(N, [200003, 5], layout, seed=N) for N, layout in ((3, 0), (8, 1))]
    want = [c.norms().copy() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.zeros(c.N, dtype=torch.float64, device="cuda") for _ in range(20)] for c in cases]
    torch.cuda.synchronize()
    for k in range(20):
        for c, s, o in zip(cases, streams, outs):
            B.wash_grad_norm(c.gpu.ctx, 0, 2, o[k], stream=s)
    torch.cuda.synchronize()
    for c, o, w in zip(cases, outs, want):
        assert all((x.cpu().numpy() == w).all() for x in o)
        c.close()


def test_refusals():
    c = Training(3, [64, 9], 0, roles="")
    ctx, norm = c.gpu.ctx, c.norm

    def refused(code, call, *args, **kw):
        before = B.wash_launch_count()
        with pytest.raises(B.WashError) as e:
            call(*args, **kw)
        assert e.value.code == code, B.wash_last_error()
        assert B.wash_launch_count() == before

    refused(B.WASH_ERR_STATE, B.wash_grad_norm, ctx, 0, 2, norm)
    refused(B.WASH_ERR_STATE, B.wash_clip_grads, ctx, 1.0, norm)
    refused(B.WASH_ERR_STATE, B.wash_sgd_step, ctx, 0.1)
    bufs = {r: torch.zeros(c.gpu.n_elems, device="cuda") for r in "pgmv"}
    c.gpu.bind(ROLES["p"], bufs["p"])
    refused(B.WASH_ERR_STATE, B.wash_sgd_step, ctx, 0.1)                                  # no gradients
    c.gpu.bind(ROLES["g"], bufs["g"])
    refused(B.WASH_ERR_STATE, B.wash_sgd_step, ctx, 0.1, 0.9)                             # no momentum stack
    c.gpu.bind(ROLES["m"], bufs["m"])
    refused(B.WASH_ERR_STATE, B.wash_adamw_step, ctx, 0, 0.1)                             # no second moments
    c.gpu.bind(ROLES["v"], bufs["v"])
    for lo, hi in ((-1, 2), (0, 3), (2, 1)):
        refused(B.WASH_ERR_ARG, B.wash_grad_norm, ctx, lo, hi, norm)
    refused(B.WASH_ERR_ARG, B.wash_grad_norm, ctx, 0, 2, None)
    refused(B.WASH_ERR_ARG, B.wash_grad_norm, ctx, 0, 2, norm.data_ptr() + 4)
    for wrong in (norm.float(), norm.long(), norm.expand(2, 3).t()):
        with pytest.raises(TypeError):
            B.wash_grad_norm(ctx, 0, 2, wrong)
    for max_norm in (-1.0, float("nan"), float("inf")):
        refused(B.WASH_ERR_ARG, B.wash_clip_grads, ctx, max_norm, norm)
        refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, 0.9, 0.0, 0, max_norm, norm)
    refused(B.WASH_ERR_ARG, B.wash_clip_grads, ctx, 1.0, None)
    refused(B.WASH_ERR_ARG, B.wash_clip_grads, ctx, 1.0, norm.data_ptr() + 4)
    for lr in (-0.1, float("nan"), 1e39):
        refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, lr)
        refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 0, lr)
    for momentum in (-0.1, 1.0, float("nan")):
        refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, momentum)
        refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 0, 0.1, momentum)
        refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 0, 0.1, 0.9, momentum)
    for eps in (0.0, -1e-8, 1e-60, float("nan")):
        refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 0, 0.1, eps=eps)
    for wd in (-0.1, float("inf")):
        refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, 0.9, wd)
    refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, 0.0, 0.0, B.WASH_STEP_NESTEROV)
    refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, 0.9, 0.0, 4)
    refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 0, 0.1, flags=B.WASH_STEP_NESTEROV)
    refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, 0.9, 0.0, B.WASH_STEP_SKIP_NONFINITE)
    refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 1 << 56, 0.1)
    c.gpu.bind(ROLES["m"], torch.zeros(c.gpu.n_elems, dtype=torch.bfloat16, device="cuda"))
    refused(B.WASH_ERR_UNSUPPORTED, B.wash_sgd_step, ctx, 0.1, 0.9)
    c.gpu.bind(ROLES["m"], bufs["g"])
    refused(B.WASH_ERR_ARG, B.wash_sgd_step, ctx, 0.1, 0.9)                               # gradients and state in one buffer
    c.gpu.bind(ROLES["m"], bufs["m"])
    c.gpu.bind(ROLES["v"], bufs["m"])
    refused(B.WASH_ERR_ARG, B.wash_adamw_step, ctx, 0, 0.1)
    with pytest.raises(B.WashError):
        B.wash_bind(ctx, 5, B.WASH_F32, bufs["p"], c.gpu.n_elems)
    with pytest.raises(B.WashError):
        B.wash_bind(ctx, B.WASH_STACK_BOTH, B.WASH_F32, bufs["p"], c.gpu.n_elems)
    for call in (B.papa_ema,):                                                            # the population operators keep to weights and first state
        refused(B.WASH_ERR_ARG, call, ctx, B.WASH_STACK_GRADS, 0.5)
    c.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_both_moments_follow_their_parameters_through_a_shuffle(layout):
    """WASH+Opt with Adam: the second moment's own context draws the same mask and permutations."""
    N = 6
    c = Training(N, RAGGED, layout, seed=14)
    moments = B.Population(N, RAGGED, layout, 0)
    moments.bind(B.WASH_STACK_OPT, c.dev["v"])
    p_layer = B.wash_layer_probs(len(RAGGED), 0.4)
    for step in range(3):
        norm = c.norms().copy()
        _step(c, "adamw", 0.9, False, step, 1.0, norm)
        B.wash_shuffle_both(c.gpu.ctx, step, 0.0, p_layer, seed=21)
        B.wash_shuffle_opt_state(moments.ctx, step, 0.0, p_layer, seed=21)
        oracle.shuffle(c.ora, c.host["p"], p_layer, seed=21, step=step, stack2=c.host["m"])
        oracle.shuffle(c.ora, c.host["v"], p_layer, seed=21, step=step)
        c.assert_equal()
    moments.close()
    c.close()


@pytest.mark.parametrize("numel", [[1] * 700, [9] * 300 + [2000] + [1] * 50, [8] * 400, [i % 7 + 1 for i in range(150)] + [30011] + [5, 5, 5]])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("N", [2, 3, 16, 37])
def test_many_tiny_tensors(N, layout, numel):
    """More tensors to a warp's coordinates, and to a lookup tile, than a lookup fetches at once."""
    c = Training(N, numel, layout, "f32", "bf16", seed=N, decay=_decay(len(numel)))
    norm = c.norms().copy()
    assert np.allclose(norm, oracle.grad_norm(c.ora, c.host["g"]), rtol=(sum(numel) + 4) * 2.0 ** -52, atol=0)
    T = len(numel)
    assert np.allclose(c.norms(T // 3, T - 2), oracle.grad_norm(c.ora, c.host["g"], T // 3, T - 2), rtol=(sum(numel) + 4) * 2.0 ** -52, atol=0)
    c.norm.copy_(torch.from_numpy(norm))
    bound = float(np.median(norm))
    _step(c, "sgd", 0.9, True, 0, bound, norm)
    _step(c, "adamw", 0.9, False, 5, bound, norm)
    B.wash_clip_grads(c.gpu.ctx, bound, c.norm)
    oracle.clip_grads(c.ora, c.host["g"], bound, norm)
    c.assert_equal()
    c.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_rows_of_every_size_near_the_kernels_choices(layout):
    """Norms at the row lengths where one block, one large block or many take a row, and just beside them."""
    for dtype in ("f32", "bf16"):
        for N in (2, 16, 48, 64):
            for P in (4095, 4096, 4104, 8192, 8200, 16384, 16392, 32768, 32776, 131072, 131080):
                if N * P > 3_000_000:
                    continue
                pop = B.Population(N, [P], layout, 0)
                g = torch.randn(pop.n_elems, device="cuda", generator=torch.Generator("cuda").manual_seed(P + N)).to(torch.float32 if dtype == "f32" else torch.bfloat16)
                pop.bind(B.WASH_STACK_GRADS, g)
                out = torch.zeros(N, dtype=torch.float64, device="cuda")
                B.wash_grad_norm(pop.ctx, 0, 1, out)
                rows = (g.view(N, -1)[:, :P] if layout == 0 else g.view(-1, N)[:P].t()).double()
                assert torch.allclose(out, rows.square().sum(1).sqrt(), rtol=2 * P * 2.0 ** -53, atol=0), (dtype, N, P)
                pop.close()


@pytest.mark.parametrize("layout", [0, 1])
def test_stacks_of_more_than_2_to_the_32_elements(layout):
    """Offsets beyond 32 bits: 64 models of 2^26 + 5 coordinates, zero but for the row's ends and two places in the middle."""
    N, P = 64, (1 << 26) + 5
    pop = B.Population(N, [P], layout, 0)
    stacks = {"p": torch.zeros(pop.n_elems, dtype=torch.bfloat16, device="cuda"), "g": torch.zeros(pop.n_elems, dtype=torch.bfloat16, device="cuda"),
              "m": torch.zeros(pop.n_elems, device="cuda")}
    for role, t in stacks.items():
        pop.bind(ROLES[role], t)

    def at(role):
        return stacks[role].view(N, pop.padded_P) if layout == 0 else stacks[role].view(pop.padded_P, N).t()

    places = [0, 1, (1 << 25) + 3, (1 << 26) - 7, P - 2, P - 1]
    values = torch.arange(1, N + 1, device="cuda", dtype=torch.float32)[:, None] * torch.tensor([1.0, 2.0, 4.0, 8.0, 16.0, 32.0], device="cuda")
    for k, e in enumerate(places):
        at("g")[:, e] = values[:, k].to(torch.bfloat16)
    at("g")[:, P:] = float("nan")                                          # padding
    norm = torch.zeros(N, dtype=torch.float64, device="cuda")
    B.wash_grad_norm(pop.ctx, 0, 1, norm)
    want = torch.stack([at("g")[:, e].double() for e in places]).square().sum(0).sqrt()
    assert torch.allclose(norm, want, rtol=1e-15, atol=0)
    B.wash_sgd_step(pop.ctx, 0.5, 0.9)
    B.wash_clip_grads(pop.ctx, float(want[20]), norm)
    torch.cuda.synchronize()
    B.wash_check(pop.ctx)
    g = values.to(torch.bfloat16).float()
    factor = torch.clamp(want[20] / (want + 1e-6), max=1.0).float()
    for k, e in enumerate(places):
        assert (at("m")[:, e] == g[:, k]).all() and (at("p")[:, e] == (-0.5 * g[:, k]).to(torch.bfloat16)).all()
        assert (at("g")[:, e] == (g[:, k] * factor).to(torch.bfloat16)).all()
    assert int((stacks["m"] != 0).sum()) == int((stacks["p"] != 0).sum()) == N * len(places)      # and nothing anywhere else
    pop.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [9000, 1_500_007])
def test_norms_of_extreme_values_in_long_rows(P, dtype, layout):
    """One infinity, one NaN, one row of the largest finite values and rows of small ones, where blocks walk several chunks."""
    N = 6
    g = torch.randn(N, P, device="cuda", generator=torch.Generator("cuda").manual_seed(P)) * 1e-3
    g[1] = 3.3e38
    g[2, P // 3] = float("inf")
    g[3, P - 1] = float("nan")
    g[4] *= 1e-37
    g[5, P // 2], g[5, P // 2 + 9] = float("-inf"), float("nan")
    g = g.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    pop = B.Population(N, [P], layout, 0)
    stack = torch.full((N, pop.padded_P), float("inf"), dtype=g.dtype, device="cuda")
    stack[:, :P] = g
    stack = (stack if layout == 0 else stack.t()).contiguous().view(-1)
    pop.bind(B.WASH_STACK_GRADS, stack)
    out = torch.zeros(N, dtype=torch.float64, device="cuda")
    B.wash_grad_norm(pop.ctx, 0, 1, out)
    want = g.double().square().sum(1).sqrt()
    assert torch.allclose(out[[0, 1, 4]], want[[0, 1, 4]], rtol=2 * P * 2.0 ** -53, atol=0)
    assert out[2] == float("inf") and out[3].isnan() and out[5].isnan()
    pop.close()


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("wdtype,gdtype", [("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("N", [2, 3, 8, 19, 64])
def test_padding_is_neither_read_nor_written(N, wdtype, gdtype, layout):
    """Padding of finite numbers, which a result would take up and a store would change: every bit of it stays, in every stack."""
    for numel in (RAGGED, ODD, [1], [4093, 2]):
        c = Training(N, numel, layout, wdtype, gdtype, seed=N, decay=_decay(len(numel)))
        real = np.zeros(c.P, bool)
        for d, o in zip(c.numel, c.off):
            real[o:o + d] = True
        pad = torch.from_numpy(np.flatnonzero(~real)).cuda()
        rows = {r: (t.view(N, c.P) if layout == 0 else t.view(c.P, N).t()) for r, t in c.dev.items()}
        for k, r in enumerate("pgmv"):
            rows[r][:, pad] = 77.0 + k
        norm = c.norms().copy()
        assert np.allclose(norm, oracle.grad_norm(c.ora, c.host["g"]), rtol=1e-12, atol=0)
        bound = 0.5 * float(norm.min())
        _step(c, "sgd", 0.9, True, 0, bound, norm)
        _step(c, "adamw", 0.9, False, 1, bound, norm)
        _step(c, "sgd", 0.0, False, 0, bound, norm)
        B.wash_clip_grads(c.gpu.ctx, bound, c.norm)
        oracle.clip_grads(c.ora, c.host["g"], bound, norm)
        for k, r in enumerate("pgmv"):
            assert (rows[r][:, pad] == 77.0 + k).all(), r
            want = W.from_stack(c.host[r], N, c.numel, c.off, c.P, layout)
            want = W.bf16_bits_to_f32(want) if want.dtype == np.uint16 else want
            assert (c.dense_of(r).view(np.uint32) == want.view(np.uint32)).all(), r
        c.close()
