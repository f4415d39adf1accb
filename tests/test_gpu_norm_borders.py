"""Gradient norms on both sides of every size at which their launch changes -- threads of a block, bytes in flight, one block or many to a row -- with the sizes
asked of the launch's own rule (csrc/wash_internal.h, compiled for the host)."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2405_17517_b200 import binding as B
from paper_2405_17517_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))
POPULATIONS = (2, 3, 8, 16, 17, 33, 47, 48, 64)
LONGEST = 1 << 20        # units of a row: beyond the last change of every population


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("rules") / "rules.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", build.CSRC, "-I", cuda, os.path.join(HERE, "optimizer_rules.cpp"), "-o", lib], check=True)
    return ctypes.CDLL(lib)


def _borders(rules, layout, N, elem_bytes, sm):
    """The last units before, and (one more) the first ones after, each change of the launch"""
    out = (ctypes.c_uint * 4)()

    def launch(units):
        rules.rule_norm(layout, N, units, elem_bytes, sm, out)
        return out[0], out[1], out[3] == 1

    def search(lo, hi):     # launches at lo and hi differ; each takes one run of sizes
        if hi - lo == 1:
            return [lo]
        mid = (lo + hi) // 2
        return (search(lo, mid) if launch(lo) != launch(mid) else []) + (search(mid, hi) if launch(mid) != launch(hi) else [])

    found = search(1, LONGEST) if launch(1) != launch(LONGEST) else []
    seen = [launch(1)] + [launch(u + 1) for u in found]
    assert len(set(seen)) == len(seen)
    return found


@pytest.mark.parametrize("sm", [132, 148])
def test_the_rule_has_borders_in_every_population(rules, sm):
    """No device needed: the search finds what the rule's text says."""
    for N in POPULATIONS:
        for elem_bytes in (2, 4):
            trip = 256 * 32 // elem_bytes                                # values of a block of 256 in a trip of 32 bytes a thread
            rows = _borders(rules, 0, N, elem_bytes, sm)
            assert {trip // 8, 2 * trip // 8} <= set(rows)               # one block to a row, 32 and 64 bytes a thread
            if N >= 48:
                assert 8 * 2 * 4 * trip // 8 in rows                     # a block of 1024 to a row
            assert len(rows) >= 3
            assert len(_borders(rules, 1, N, elem_bytes, sm)) >= (2 if N <= 16 else 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("N", POPULATIONS)
def test_norms_at_the_borders(rules, N, layout, dtype):
    sm = torch.cuda.get_device_properties(0).multi_processor_count
    for border in _borders(rules, layout, N, 4 if dtype == "f32" else 2, sm):
        for P in (8 * border - 3, 8 * border, 8 * border + 1, 8 * border + 8):
            pop = B.Population(N, [P], layout, 0)
            values = torch.randn(N, P, device="cuda", generator=torch.Generator("cuda").manual_seed(P + N)).to(torch.float32 if dtype == "f32" else torch.bfloat16)
            stack = torch.full((N, pop.padded_P), 1e6, dtype=values.dtype, device="cuda")          # padding that a sum would show
            stack[:, :P] = values
            stack = (stack if layout == 0 else stack.t()).contiguous().view(-1)
            pop.bind(B.WASH_STACK_GRADS, stack)
            out = torch.zeros(N, dtype=torch.float64, device="cuda")
            for _ in range(2):                                           # the second one finds what the first one left of the report
                out.fill_(-1.0)
                B.wash_grad_norm(pop.ctx, 0, 1, out)
                # squares are exact in binary64, sums of non-negative terms off by P 2^-53 at most, on either side; the root halves it
                assert torch.allclose(out, values.double().square().sum(1).sqrt(), rtol=2 * P * 2.0 ** -53, atol=0), (P, border)
            B.wash_check(pop.ctx)
            pop.close()
