"""Fine-tuning on tokens: the ends of a small language model trained first-order, then ZO steps of a stack between them.

    python examples/token_steps.py

A sequence whose next token follows from the present one is learnt twice: by the tied table and the norm alone (exact
gradients, plain SGD), and then, with new rules for a part of the vocabulary, by the coefficients of the 256-wide toy graph
(Algorithm 2, two-sided) with the ends frozen.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2607_01125_gb300 as zo
from paper_2607_01125_gb300.model import AdaptedLinear, TokenStep, ZOStep, calibrate_bases, coefficient_offsets
from synth import normal, tensor_seed, workload


def main(warm_steps=60, zo_steps=150, vocab=500, dev="cuda:0"):
    """(losses of the first-order steps, L+ of the ZO steps)."""
    w = workload("toy_fp32", lr=2e-3)
    ctx = zo.Context(0)
    rng = torch.Generator().manual_seed(1)
    follows = torch.randperm(vocab, generator=rng)

    def batch(rule, T=w.T):
        ids = torch.randint(0, vocab, (T,), generator=rng)
        targets = rule[ids]
        targets[torch.rand(T, generator=rng) < 0.05] = -100          # padding: not counted
        return ids.to(dev), targets.to(dev)

    table = normal((vocab, w.d_model), 11, dev, std=0.1)
    head = normal((vocab, w.d_model), 12, dev, std=0.1)
    gain, bias = torch.ones(w.d_model, device=dev), torch.zeros(w.d_model, device=dev)
    ends = TokenStep(None, table, head=head, gain=gain, bias=bias, ctx=ctx)
    first = []
    for _ in range(warm_steps):
        ids, targets = batch(follows, 1024)
        ends.forward(ids)
        first.append(ends.ends_grad(ids, targets).clone())
        for p, g, lr in ((table, ends.dtable, 1.0), (head, ends.dhead, 1.0), (gain, ends.dgain, 0.1), (bias, ends.dbias, 0.1)):
            p.sub_(g, alpha=lr)

    specs = w.linears()
    lins = []
    for s, off in zip(specs, coefficient_offsets(specs, w.r)):
        W = torch.eye(s.d_out, s.d_in, device=dev) + normal((s.d_out, s.d_in), tensor_seed(w, "W", s.name), dev, std=0.01)
        U = torch.empty(s.d_in, w.r, device=dev)
        lins.append(AdaptedLinear(s.name, W, U, s.layer_id, off, w.r))
    ids, _ = batch(follows, w.n_cal)
    x = torch.empty(w.n_cal, w.d_model, device=dev)
    zo.zoact_embed(ctx, table, ids, x)
    U0 = [normal(l.U.shape, 20 + l.layer_id, dev) for l in lins]
    for l, u in zip(lins, U0):
        l.U.copy_(u)
    calibrate_bases(ctx, ZOStep(ctx, w.kind, lins, w.n_cal, w.act_dtype), x, w.r)
    stack = ZOStep(ctx, w.kind, lins, w.T, w.act_dtype, eps=1e-2, lr=w.lr)
    model = TokenStep(stack, table, head=head, gain=gain, bias=bias)
    ids, targets = batch(follows.roll(1))                            # one batch, other rules
    second = [model.step(ids, targets, i + 1, seed=7, query=i).clone() for i in range(zo_steps)]
    torch.cuda.synchronize()
    status = ctx.device_status()
    if status != 0:
        raise RuntimeError(f"device status {status}")
    ctx.close()
    return [float(v) for v in first], [float(v[0]) for v in second]


if __name__ == "__main__":
    first, second = main()
    print("first-order steps of the ends: loss %.4f -> %.4f" % (first[0], first[-1]))
    print("ZO steps of the stack:         loss %.4f -> %.4f" % (second[0], sum(second[-10:]) / 10))
