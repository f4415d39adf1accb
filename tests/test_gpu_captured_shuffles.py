"""Shuffles captured into graphs, next to eager calls and steps of the same context: a graph keeps the probabilities it was captured with, an eager call its
own, and the multipliers of wash_set_decay are those set last, whatever is replayed in between."""
import numpy as np
import pytest
import torch

import oracle
from paper_2405_17517_b200 import binding as B
from paper_2405_17517_b200 import workloads as W
from gpu_util import Case, bits, to_device, to_host_bits

pytestmark = pytest.mark.gpu

NUMEL = [2500, 33, 7, 4096, 1]


class Step:
    """Weights, gradients and momentum of a population on both sides."""

    def __init__(self, N, layout):
        self.c = Case(N, NUMEL, layout, "f32", "f32", seed=N)
        self.ctx = self.c.gpu.ctx
        grads = W.flat_population(N, sum(NUMEL), seed=77, std=0.02)
        self.host_g = W.to_stack(grads, NUMEL, self.c.off, self.c.P, layout)
        self.dev_g = to_device(self.host_g)
        self.c.gpu.bind(B.WASH_STACK_GRADS, self.dev_g)

    def both(self, oracle_only, decay, p, step, seed=3):
        """a step of SGD and a shuffle of weights and momentum"""
        if not oracle_only:
            B.wash_sgd_step(self.ctx, 0.1, 0.9, 0.05)
            B.wash_shuffle_both(self.ctx, step, 0.0, p, seed=seed)
        if oracle_only is not None:
            oracle.sgd_step(self.c.ora, self.c.host, self.host_g, self.c.host_opt, 0.1, 0.9, 0.05, decay=decay)
            oracle.shuffle(self.c.ora, self.c.host, p, seed=seed, step=step, stack2=self.c.host_opt)

    def assert_equal(self):
        torch.cuda.synchronize()
        B.wash_check(self.ctx)
        assert_same(self.c.dev, self.c.host)
        assert_same(self.c.dev_opt, self.c.host_opt)


def assert_same(dev, host):
    bad = np.flatnonzero((to_host_bits(dev) != bits(host)) & ~np.isnan(np.ascontiguousarray(host).reshape(-1)))    # padding is NaN
    assert bad.size == 0, "%d elements differ, first at %d" % (bad.size, bad[0])


def captured(record):
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        record()
    return graph


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("N", [2, 5, 24])
def test_a_replayed_shuffle_leaves_the_decay_multipliers_alone(N, layout):
    """A step and a shuffle in one graph, with probabilities that no call had before; the multipliers change between the replays."""
    s = Step(N, layout)
    p = np.array([0.3, 0.1, 0.9, 0.2, 1.0])
    decay = [1.0, 0.0, 0.5, 2.0, 0.25]
    B.wash_set_decay(s.ctx, decay)
    graph = captured(lambda: s.both(None, None, p, 4))
    for decay in (decay, [0.0, 1.0, 3.0, 0.5, 0.125], [4.0, 0.25, 0.0, 1.0, 2.0], [4.0, 0.25, 0.0, 1.0, 2.0], None):
        B.wash_set_decay(s.ctx, decay)
        for eager in (False, True, False):
            if eager:
                s.both(False, decay, p, 4)
            else:
                graph.replay()
                s.both(True, decay, p, 4)
            s.assert_equal()
    s.c.close()


@pytest.mark.parametrize("mode", [B.WASH_MODE_STREAM, B.WASH_MODE_SPARSE, B.WASH_MODE_AUTO], ids=["stream", "sparse", "auto"])
@pytest.mark.parametrize("layout", [0, 1])
def test_graphs_and_eager_calls_keep_their_own_probabilities(layout, mode):
    """Two graphs captured with probabilities that no call had before, one of them with those of the other's last call, and eager calls with the same and with
    many other probabilities before, between and behind the replays."""
    N = 6
    c = Case(N, NUMEL, layout, "f32", None, seed=2)
    B.wash_set_mode(c.gpu.ctx, mode)
    layers = np.array([0.25, 1.0, 0.0, 0.03, 0.5])
    recorded = [[(0.3, None, 1), (0.0, layers, 2)], [(0.0, layers, 3), (0.015, None, 4)]]
    want, step = [0, 0], 100

    def expect(p, layer, at):
        got = oracle.shuffle(c.ora, c.host, p if layer is None else layer, seed=9, step=at)
        want[0] += got[0]
        want[1] += got[1]

    def record(calls):
        for p, layer, at in calls:
            B.wash_shuffle(c.gpu.ctx, at, p, layer, seed=9, stats=c.stats_dev)

    graphs = [captured(lambda calls=calls: record(calls)) for calls in recorded]
    for turn in range(3):
        for p, layer in ((0.3, None), (0.0, layers), (0.015, None), (0.9, None), (0.2, None), (0.5, None), (0.7, None), (0.5, None), (0.015, None)):
            for eager in range(2):
                B.wash_shuffle(c.gpu.ctx, step, p, layer, seed=9, stats=c.stats_dev)
                expect(p, layer, step)
                step += 1
                if eager == 0:
                    graphs[step % 2].replay()
                    for call in recorded[step % 2]:
                        expect(*call)
            torch.cuda.synchronize()
            assert_same(c.dev, c.host)
    B.wash_check(c.gpu.ctx)
    assert c.gpu_stats() == tuple(want)
    c.close()


def test_a_captured_call_of_refused_probabilities_leaves_the_capture_intact():
    c = Case(4, NUMEL, 0, "f32", None, seed=5)

    def record():
        with pytest.raises(B.WashError) as e:
            B.wash_shuffle(c.gpu.ctx, 1, 1.5, None, seed=1)
        assert e.value.code == B.WASH_ERR_ARG
        with pytest.raises(B.WashError):
            B.wash_shuffle(c.gpu.ctx, 1, 0.0, [0.1, 0.2, float("nan"), 0.1, 0.1], seed=1)
        B.wash_shuffle(c.gpu.ctx, 1, 0.4, None, seed=1)

    graph = captured(record)
    graph.replay()
    oracle.shuffle(c.ora, c.host, 0.4, seed=1, step=1)
    torch.cuda.synchronize()
    assert_same(c.dev, c.host)
    c.close()


def test_the_other_operators_in_a_graph_with_a_shuffle():
    """The pull toward the mean, the average and the distance to the consensus behind a captured shuffle, with the statistic in the shuffle's pass, too."""
    c = Case(5, NUMEL, 0, "f32", None, seed=6)
    avg = torch.zeros(c.P, device="cuda")
    sq, inside = torch.zeros(5, dtype=torch.float64, device="cuda"), torch.zeros(5, dtype=torch.float64, device="cuda")

    def record():
        B.wash_shuffle_consensus(c.gpu.ctx, B.WASH_STACK_PARAMS, 8, 0.6, None, 1, tensor_bounds=(0, len(NUMEL)), dev_sq_out=inside)
        B.papa_ema(c.gpu.ctx, B.WASH_STACK_PARAMS, 0.75)
        B.population_average(c.gpu.ctx, B.WASH_STACK_PARAMS, avg, B.WASH_F32)
        B.wash_consensus_sq(c.gpu.ctx, B.WASH_STACK_PARAMS, 0, len(NUMEL), sq)

    graph = captured(record)
    want = np.zeros(c.P, np.float32)
    for _ in range(2):
        B.wash_shuffle(c.gpu.ctx, 20, 0.1, None, seed=1)
        oracle.shuffle(c.ora, c.host, 0.1, seed=1, step=20)
        sq.zero_()
        inside.zero_()
        graph.replay()
        before = oracle.consensus_sq(c.ora, c.host)
        oracle.shuffle(c.ora, c.host, 0.6, seed=1, step=8)
        oracle.papa_ema(c.ora, c.host, 0.75)
        oracle.population_average(c.ora, c.host, want)
        torch.cuda.synchronize()
        assert_same(c.dev, c.host)
        assert_same(avg, want)
        # both sides add binary64 squares of differences that are exact to a few units: n additions in any order
        rtol = 8 * sum(NUMEL) * 2.0 ** -53
        assert np.allclose(inside.cpu().numpy(), before, rtol=rtol, atol=0)
        assert np.allclose(sq.cpu().numpy(), oracle.consensus_sq(c.ora, c.host), rtol=rtol, atol=0)
    c.close()


def test_a_captured_plan_of_the_one_model_per_device_form_keeps_its_probabilities():
    N = 4
    ctx = B.wash_create(N, NUMEL)
    P = B.wash_stack_elems(ctx, len(NUMEL))[0]
    row = torch.zeros(P, device="cuda")
    B.wash_exchange_bind(ctx, 1, B.WASH_STACK_PARAMS, B.WASH_F32, row, P)

    def eager(p):
        B.wash_exchange_plan(ctx, 6, p, None, seed=2)
        return B.wash_exchange_counts(ctx, N)

    graph = captured(lambda: B.wash_exchange_plan(ctx, 6, 0.35, None, seed=2))
    want = eager(0.35)
    others = [0.1, 0.5, 0.7, 0.9, 0.2, 0.05]
    assert len({eager(p)[1] for p in others} | {want[1]}) == 7
    for p in others:
        other = eager(p)
        graph.replay()
        assert B.wash_exchange_counts(ctx, N) == want
        assert eager(p) == other
    B.wash_destroy(ctx)
