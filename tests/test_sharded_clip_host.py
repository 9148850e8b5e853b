"""CPU: what the clipping of a sharded model gathers and hands to the library, on two gloo ranks and on one without a process
group; a recording stand-in takes the library's place."""
import os
import socket

import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2504_05295_b200 import sharded


def _free_port():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        return s.getsockname()[1]


class _Recording:
    """Lists are numbers here: the norm of a list."""

    def __init__(self, log):
        self.log = log

    def grad_norm(self, items, norm_type=2, norm_out=None, stream=None):
        self.log.append(("norm", items, norm_type))
        norm_out.fill_(items)

    def clip_grads(self, items, max_norm, norms=None, norm_type=2, norm_out=None, coef_out=None, stream=None):
        self.log.append(("clip", items, max_norm, norms.tolist(), norm_type))
        if norm_out is not None:
            norm_out.fill_(norms.norm())
            coef_out.fill_(max_norm / norms.norm())


def _worker(rank, world, port, out):
    os.environ["MASTER_ADDR"], os.environ["MASTER_PORT"] = "127.0.0.1", str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    log = []
    clipper = sharded.ShardedClipper(_Recording(log), float(rank + 2), 6.0, "cpu")
    clipper.clip(1.0)
    clipper.clip(2.0, "inf", scale_whole=False)
    out[rank] = (log, float(clipper.norm), float(clipper.coef))
    dist.destroy_process_group()


def test_two_ranks_clip_by_the_norm_of_all():
    world, port = 2, _free_port()
    with mp.Manager() as mgr:
        out = mgr.dict()
        mp.spawn(_worker, args=(world, port, out), nprocs=world, join=True)
        seen = [out[r] for r in range(world)]
    norms = [2.0, 3.0, 6.0]      # the ranks' shards in their order, then what all hold, once
    for rank, (log, norm, coef) in enumerate(seen):
        mine = float(rank + 2)
        assert log == [("norm", mine, 2), ("norm", 6.0, 2), ("clip", mine, 1.0, norms, 2), ("clip", 6.0, 1.0, norms, 2),
                       ("norm", mine, "inf"), ("norm", 6.0, "inf"), ("clip", mine, 2.0, norms, "inf")]
        assert norm == 7.0 and abs(coef - 2.0 / 7.0) < 1e-6
    assert seen[0][1:] == seen[1][1:]


def test_one_rank_needs_no_process_group():
    log = []
    clipper = sharded.ShardedClipper(_Recording(log), 5.0, device="cpu")
    clipper.clip(1.0)
    assert log == [("norm", 5.0, 2), ("clip", 5.0, 1.0, [5.0], 2)]
    assert float(clipper.norm) == 5.0
