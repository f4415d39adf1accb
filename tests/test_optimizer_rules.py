"""The sizes of the optimizer side's launches (csrc/wash_internal.h), compiled for the host and evaluated over their ranges."""
import ctypes
import os
import subprocess

import pytest

from paper_2405_17517_b200 import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("rules") / "rules.so")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc()))), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I", build.CSRC, "-I", cuda, os.path.join(HERE, "optimizer_rules.cpp"), "-o", lib], check=True)
    L = ctypes.CDLL(lib)
    L.rule_norm_partials.restype = ctypes.c_ulonglong
    return L


SIZES = sorted({max(1, (1 << k) + d) for k in range(0, 31) for d in (-1, 0, 1, 77)} | set(range(1, 300)) | {(1 << 30) - 1})


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("elem_bytes", [2, 4])
def test_a_norms_launch_covers_the_range_and_its_partial_sums_fit(rules, layout, elem_bytes):
    """Every unit is in a chunk, every block has one, no block starts behind the last one, kernels exist for the sizes, counters stay
    within 32 bits, and the blocks' partial sums fit the context's buffer -- on devices of 1 to 200 SMs, for rows up to the longest."""
    out = (ctypes.c_uint * 4)()
    for sm in (1, 2, 16, 132, 148, 200):
        for N in (2, 3, 5, 8, 15, 16, 17, 31, 33, 47, 48, 63, 64):
            room = rules.rule_norm_partials(layout, N, sm)
            for units in SIZES:
                if units >= 1 << 30:
                    continue
                rules.rule_norm(layout, N, units, elem_bytes, sm, out)
                threads, together, chunks, per_model = out
                assert threads in ((256, 1024) if layout == 0 else (256, 512))
                assert together * 8 * elem_bytes in (32, 64)
                per_chunk = threads if layout == 0 else threads // N
                assert per_chunk >= 1 and (chunks - 1) * per_chunk < units <= chunks * per_chunk
                assert 1 <= per_model and (per_model - 1) * together < chunks
                assert per_model == 1 or per_model * N <= room
                assert (chunks + (per_model + 1) * together) * per_chunk < 1 << 32
                assert per_model * (N if layout == 0 else 1) < 1 << 31


def test_an_empty_range_is_a_launch_that_finds_nothing(rules):
    out = (ctypes.c_uint * 4)()
    for layout in (0, 1):
        for N in (2, 17, 64):
            rules.rule_norm(layout, N, 0, 4, 148, out)
            assert out[2] == 0 and out[3] == 1


def test_a_chunk_holds_whole_units_of_all_models(rules):
    for N in range(2, 65):
        assert rules.rule_chunk_units(0, N) == 256
        units = rules.rule_chunk_units(1, N)
        assert 1 <= units and 256 - N < units * N <= 256      # an octet a thread, the same models in every chunk
