"""The example's sum over ranks, on two processes with CPU tensors."""
import os
import sys

import torch
import torch.distributed as dist
import torch.multiprocessing as mp

EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


def _rank(rank, store):
    sys.path.insert(0, EXAMPLES)
    from decoder_block import sum_over_ranks
    dist.init_process_group("gloo", init_method=f"file://{store}", rank=rank, world_size=2)
    t = torch.full((3, 8), 1.0 + rank, dtype=torch.bfloat16)
    sum_over_ranks(t)
    dist.destroy_process_group()
    assert bool((t == 3.0).all())


def test_every_rank_gets_the_sum(tmp_path):
    mp.spawn(_rank, args=(str(tmp_path / "store"),), nprocs=2)
