"""Clipped steps of a population that is cut along its coordinates: every rank adds up the squares of its own shard, one all-reduce of N numbers gives the norms,
and the ranks' steps together are the step of the whole.  Two and three CPU ranks over gloo, with the oracle in the library's place."""
import os

import numpy as np
import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

import oracle
from paper_2405_17517_b200 import sharding
from paper_2405_17517_b200 import workloads as W
from test_sharding_gloo import _free_port

NUMEL = [4001, 64, 7, 1200, 3, 36, 2048]
DECAY = [1.0, 0.0, 1.0, 0.5, 0.0, 1.0, 0.25]
N = 4


def _rank_main(rank, world, port, out_dir):
    os.environ["MASTER_ADDR"] = "127.0.0.1"
    os.environ["MASTER_PORT"] = str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    try:
        full = [W.flat_population(N, sum(NUMEL), seed=30 + k, std=s) for k, s in enumerate((0.05, 0.02, 0.01))]      # weights, gradients, momentum
        segs = sharding.plan_shards(NUMEL, world)[rank]
        numel, tensor_id, coord_begin = sharding.segment_arrays(segs)
        mine = [np.ascontiguousarray(np.concatenate([a[:, c] for c in sharding.dense_slices(NUMEL, segs)], axis=1)) for a in full]
        pop = oracle.Population(N, numel, tensor_id=tensor_id, coord_begin=coord_begin)
        squares = torch.from_numpy(oracle.grad_norm(pop, mine[1]) ** 2)
        dist.all_reduce(squares)
        norm = squares.sqrt().numpy()
        bound = float(np.median(norm))
        oracle.sgd_step(pop, mine[0], mine[1], mine[2], 0.1, 0.9, 0.02, sharding.segment_probs(DECAY, segs), max_norm=bound, norm=norm)
        gathered = [None] * world
        dist.all_gather_object(gathered, (segs, mine[0], mine[2], norm))
        if rank == 0:
            whole = oracle.Population(N, NUMEL)
            assert np.allclose(norm, oracle.grad_norm(whole, full[1]), rtol=1e-13, atol=0)
            got = [a.copy() for a in (full[0], full[2])]
            for segs_r, p, m, norm_r in gathered:
                assert (norm_r == norm).all()
                at = 0
                for c in sharding.dense_slices(NUMEL, segs_r):
                    w = c.stop - c.start
                    got[0][:, c], got[1][:, c] = p[:, at:at + w], m[:, at:at + w]
                    at += w
            oracle.sgd_step(whole, full[0], full[1], full[2], 0.1, 0.9, 0.02, DECAY, max_norm=bound, norm=norm)
            ok = all((a.view(np.uint32) == b.view(np.uint32)).all() for a, b in zip(got, (full[0], full[2])))
            with open(os.path.join(out_dir, "result.txt"), "w") as f:
                f.write("ok" if ok else "mismatch")
        dist.barrier()
    finally:
        dist.destroy_process_group()


@pytest.mark.parametrize("world", [2, 3])
def test_clipped_steps_of_shards(world, tmp_path):
    oracle.build()
    mp.spawn(_rank_main, args=(world, _free_port(), str(tmp_path)), nprocs=world, join=True)
    assert (tmp_path / "result.txt").read_text() == "ok"
