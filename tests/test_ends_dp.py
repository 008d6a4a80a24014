"""World-size-2 check (gloo, CPU) of clipping over ranks: which gradients a rank counts, the exchange of the sums, the factor that all ranks get.  The two
calls that run on the GPU are stood in for by the same arithmetic in torch."""
import math
import os
import socket

import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2509_25149_b200 import dp


class FakeList:
    def __init__(self, grads, outs=None):
        self.grads, self.outs = list(grads), list(outs) if outs is not None else list(grads)


def fake_binding():
    from paper_2509_25149_b200 import binding as B

    B.grad_list = FakeList
    B.nvfp4_grad_sq_norm_workspace_bytes = lambda: 256

    def sq_norm(held, total, workspace, accumulate=False):
        total.copy_(sum(g.double().square().sum() for g in held.grads).reshape(1))

    def clip(held, total, most, stats):
        norm = math.sqrt(float(total))
        factor = most / norm if norm > most else 1.0
        stats.copy_(torch.tensor([norm, factor]))
        for g, o in zip(held.grads, held.outs):
            o.copy_(g * factor)

    B.nvfp4_grad_sq_norm, B.nvfp4_grad_clip = sq_norm, clip


def _worker(rank, world, port, out):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    try:
        fake_binding()
        whole = torch.arange(1.0, 25.0).view(6, 4)
        gain = torch.tensor([3.0, -2.0])
        b, e = dp.weight_grad_shard(6, rank, world)
        shard, own_gain, kept = whole[b:e].clone(), gain.clone(), torch.zeros(e - b, 4)
        norm = math.sqrt(float(whole.square().sum() + gain.square().sum()))
        clipper = dp.GradClipper([shard], 0.5 * norm, outs=[kept], sharded=True, replicated=[own_gain])
        stats = clipper()
        assert torch.allclose(stats, torch.tensor([norm, 0.5]), rtol=1e-6)
        assert torch.allclose(kept, 0.5 * whole[b:e]) and torch.equal(shard, whole[b:e]) and torch.allclose(own_gain, 0.5 * gain)
        # gradients that every rank has in full: no exchange, and the same factor everywhere
        full = whole.clone()
        stats = dp.GradClipper([full], 1e6)()
        assert abs(float(stats[0]) - math.sqrt(float(whole.square().sum()))) < 1e-3 and torch.equal(full, whole)
        # a rank without a share of its own, beside replicated gradients that the other one counts
        nothing = dp.GradClipper([], 1e6, sharded=True, replicated=[gain.clone()])
        stats = nothing()
        assert abs(float(stats[0]) - math.sqrt(13.0)) < 1e-6
        out.put((rank, "ok"))
    finally:
        dist.destroy_process_group()


def test_clipping_over_two_ranks():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    ctx = mp.get_context("spawn")
    out = ctx.Queue()
    ranks = [ctx.Process(target=_worker, args=(r, 2, port, out)) for r in range(2)]
    for p in ranks:
        p.start()
    for p in ranks:
        p.join(120)
        assert p.exitcode == 0
    assert sorted(out.get(timeout=5) for _ in ranks) == [(0, "ok"), (1, "ok")]
