"""Data-parallel losses on tokens across 2 CPU ranks (gloo): ranks with different numbers of rows that have a target.

The loss vectors are means over the counted rows, so the ranks weigh theirs by their share of these before dp.allreduce_loss
averages them; the result is the vector of the whole batch, which the plain average is not.
"""
import os
import socket

import numpy as np
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from oracle import ends

T, EPS = 20, 1e-2


def _shard(rank):
    """Hidden states of both signs, the head and the targets of a rank: 15 counted rows on the first, 4 on the second."""
    rng = np.random.default_rng(rank)
    W = np.random.default_rng(9).standard_normal((30, 6))
    H = rng.standard_normal((T, 6))
    t = rng.integers(0, 30, T)
    t[:5 if rank == 0 else 16] = -100
    return np.concatenate([H + EPS * rng.standard_normal(H.shape), H - EPS * rng.standard_normal(H.shape)]), W, t


def _vector(H, W, t):
    loss, _, L = ends.cross_entropy(H, W, t, 2)
    return ends.pair(L, loss, t, EPS)


def _worker(rank, world, port, q):
    os.environ["MASTER_ADDR"] = "127.0.0.1"
    os.environ["MASTER_PORT"] = str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    from paper_2607_01125_gb300.dp import allreduce_loss
    H, W, t = _shard(rank)
    targets, out = torch.from_numpy(t), torch.from_numpy(_vector(H, W, t))
    n = (targets >= 0).sum().double()
    total = n.clone()
    dist.all_reduce(total)
    out.mul_(n * (world / total.clamp(min=1)))
    allreduce_loss(out, finish=lambda v, w: v.div_(w))
    q.put((rank, out.numpy().tolist()))
    dist.destroy_process_group()


def test_ranks_with_different_numbers_of_targets():
    s = socket.socket()
    s.bind(("127.0.0.1", 0))
    port = s.getsockname()[1]
    s.close()
    ctx = mp.get_context("spawn")
    q = ctx.Queue()
    procs = [ctx.Process(target=_worker, args=(r, 2, port, q)) for r in range(2)]
    for p in procs:
        p.start()
    results = [q.get(timeout=120) for _ in procs]
    for p in procs:
        p.join(timeout=60)
        assert p.exitcode == 0
    (Ha, W, ta), (Hb, _, tb) = _shard(0), _shard(1)
    whole = _vector(np.concatenate([Ha[:T], Hb[:T], Ha[T:], Hb[T:]]), W, np.concatenate([ta, tb]))
    plain = (_vector(Ha, W, ta) + _vector(Hb, W, tb)) / 2
    assert np.abs(plain - whole)[:2].min() > 1e-2 * whole[0]
    for _, out in results:
        np.testing.assert_allclose(out, whole, rtol=1e-12, atol=1e-12)
