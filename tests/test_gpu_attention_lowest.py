"""Keys that are hidden by their values: a column of the type's lowest value against positive queries makes scores of -infinity in fp32.
Rows with other keys go by those; rows without have an output and gradients of 0, as where a mask leaves nothing.
(fp16's lowest value makes no score of -infinity.)"""
import pytest
import torch

from test_gpu_attention import TYPES, Case, clean, ctx, packed  # noqa: F401  (ctx: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 128, 33])
@pytest.mark.parametrize("causal", [True, False])
def test_keys_of_the_lowest_value(ctx, dt, d, causal):  # noqa: F811
    lens = (40, 200, 7, 129)
    c = Case(ctx, dt, 4, 2, d, packed(*lens), causal, grad=True)
    low = torch.finfo(TYPES[dt]).min
    c.q[:, ::d] = 64.0                                        # positive against the lowest: -infinity
    c.k[:, ::d] = 0.0                                         # (the others: no part of the scores)
    first = lens[0]
    c.k[first:first + lens[1], ::d] = low                     # the second sequence: all keys
    late = first + lens[1] + lens[2] + 60
    c.k[late:late + 20, ::d] = low                            # the last one: keys 60 to 79
    c.forward()
    outs = c.grads()
    clean(ctx)
    none = slice(first, first + lens[1])
    assert (c.O[none] == 0).all() and (c.lse[none] == -float("inf")).all()
    for t in outs:
        assert torch.isfinite(t).all() and (t[none] == 0).all()
    # the other sequences as without them
    for i, n in ((0, 40), (2, 7)):
        at = sum(lens[:i])
        alone = Case(ctx, dt, 4, 2, d, packed(n), causal, grad=True)
        for name in ("q", "k", "v", "dO"):
            getattr(alone, name).copy_(getattr(c, name)[at:at + n])
        alone.forward()
        got = alone.grads()
        clean(ctx)
        alone.check_forward()
        alone.check_grads(got)
        assert torch.equal(alone.O, c.O[at:at + n]) and all(torch.equal(a, b[at:at + n]) for a, b in zip(got, outs))
    # hidden keys have no part in anything, and what is left is what the keys without them give
    assert (outs[1][late:late + 20] == 0).all() and (outs[2][late:late + 20] == 0).all()
    if not causal:
        at = late - 60
        keys = [i for i in range(129) if not 60 <= i < 80]
        alone = Case(ctx, dt, 4, 2, d, [(0, 129, 0, 109)], False, grad=True)
        alone.q.copy_(c.q[at:])
        alone.dO.copy_(c.dO[at:])
        for name in ("k", "v"):
            getattr(alone, name).copy_(getattr(c, name)[at:][keys])
        alone.forward()
        got = alone.grads()
        clean(ctx)
        alone.check_forward()
        alone.check_grads(got)
        alone.check_grads([outs[0][at:], outs[1][at:][keys], outs[2][at:][keys]])
