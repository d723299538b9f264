"""The gradient by keys that very many rows see, on the CUDA cores: rows of work of dk and dv that are cut nowhere (heads wider than
128) and run through their rows in runs of 4096 positions, with lengths around that and heads of a group.

Counted in 32 bits over a whole row of work, 2^24 positions of 128 heads were 2^31 rows: none.  (Such a call takes minutes, so its
count is bounded where the kernel is compiled; here the runs' borders are tested.)"""
import pytest

from test_gpu_attention import Case, clean, ctx, packed  # noqa: F401  (ctx: fixture)
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n", [4095, 4096, 4097, 8200])
def test_causal_rows_around_a_run(ctx, dt, n):  # noqa: F811
    c = Case(ctx, dt, 1, 1, 136, packed(7, n), grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_grads(outs)
    again = c.grads()
    clean(ctx)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("heads", [3, 71])
def test_groups_of_many_rows(ctx, dt, heads):  # noqa: F811
    """Runs of 3 and 71 heads a position on few keys, some of them behind a queries' start."""
    for causal, span in ((False, (0, 9000, 0, 40)), (True, (0, 4200, 0, 4203))):
        if heads == 71 and causal:
            continue
        c = Case(ctx, dt, heads, 1, 130, [span], causal, grad=True)
        c.forward()
        outs = c.grads()
        clean(ctx)
        c.check_grads(outs)
