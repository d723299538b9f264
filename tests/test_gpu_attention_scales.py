"""The gradient of attention in fp16: what is rounded to fp16 on the way is scaled for each sequence and key head by itself, so that large
values in one leave the bits of the others as they were."""
import pytest
import torch

import paper_2607_01125_gb300 as zo
from test_gpu_attention import Case, clean, ctx, packed  # noqa: F401  (ctx: fixture)

pytestmark = pytest.mark.gpu
LENS = (33, 100, 1, 70, 160)                          # short: rows of work are cut nowhere, packed or alone


def rows(t, i):
    first = sum(LENS[:i])
    return t[first:first + LENS[i]]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,d", [(4, 2, 64), (8, 1, 128), (2, 2, 24), (4, 4, 128)])
@pytest.mark.parametrize("large", [1, 4])
def test_a_sequence_of_large_values_leaves_the_others(ctx, heads, kv_heads, d, large, causal):  # noqa: F811
    c = Case(ctx, "fp16", heads, kv_heads, d, packed(*LENS), causal, grad=True)
    rows(c.dO, large).mul_(2.0 ** 7)
    rows(c.v, large).mul_(2.0 ** 10)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    for i, n in enumerate(LENS):
        alone = Case(ctx, "fp16", heads, kv_heads, d, packed(n), causal, grad=True)
        for name in ("q", "k", "v", "dO", "O", "lse"):
            getattr(alone, name).copy_(rows(getattr(c, name), i))
        got = alone.grads()
        clean(ctx)
        if i != large:                                # (its gradients pass fp16's 65504)
            alone.check_grads(got)
        for name, a, b in zip(("dq", "dk", "dv"), got, outs):
            assert torch.equal(a, rows(b, i)), (name, i)


def test_a_key_head_of_large_values_leaves_the_others(ctx):  # noqa: F811
    got = []
    for power in (0, 9):
        c = Case(ctx, "fp16", 6, 3, 64, packed(*LENS), grad=True)
        c.dO[:, 128:256] *= 2.0 ** (power // 2)                             # the second key head's query heads
        c.v[:, 64:128] *= 2.0 ** power
        c.forward()
        outs = c.grads()
        clean(ctx)
        c.check_grads(outs)
        got.append([torch.cat([t[:, :n], t[:, 2 * n:]], dim=1) for t, n in zip(outs, (128, 64, 64))])
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_many_sequences_of_different_sizes(ctx):  # noqa: F811
    """Sequences whose gradients' sizes differ by powers of two up to 2^24, each with its own digits, twice with one plan."""
    lens = [5, 0, 17, 40] * 40
    c = Case(ctx, "fp16", 4, 2, 64, packed(*lens), grad=True)
    first = 0
    for i, n in enumerate(lens):
        small = c.dO[first:first + n].float() * 2.0 ** (i % 13 - 8)
        c.dO[first:first + n] = torch.where(small.abs() < 2.0 ** -14, torch.zeros_like(small), small).half()
        c.v[first:first + n] *= 2.0 ** (i % 11)
        first += n
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_grads(outs)
    again = c.grads()
    clean(ctx)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
