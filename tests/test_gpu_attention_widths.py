"""Attention and its gradient on the tensor cores where a tile's rows or keys end inside of a warp and a head's columns inside of what a
thread stores at a time: every way out of the kernels (whole rows of work, halves of the keys joined, parts joined), in widths
that are multiples of 8 and nothing more."""
import pytest

from test_gpu_attention import Case, clean, ctx, packed  # noqa: F401  (ctx: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [8, 16, 72, 104, 120, 128])
@pytest.mark.parametrize("heads,kv_heads", [(5, 1), (3, 3)])
def test_rows_that_end_inside_of_a_warp(ctx, dt, d, heads, kv_heads):  # noqa: F811
    """Whole rows of work and halves of the keys, causal or not."""
    for causal in (True, False):
        spans = [(0, 13, 0, 13), (13, 7, 13, 300), (20, 1, 313, 129), (21, 150, 442, 150), (171, 29, 592, 1), (200, 41, 593, 777)]
        c = Case(ctx, dt, heads, kv_heads, d, spans, causal, grad=True)
        c.forward()
        outs = c.grads()
        clean(ctx)
        c.check_forward()
        c.check_grads(outs)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [8, 72, 104, 128])
def test_cut_rows_that_end_inside_of_a_warp(ctx, dt, d):  # noqa: F811
    """13 positions of 5 heads on 5000 keys (forward and dq are cut along the keys), 37 keys that 3000 rows see (dk and dv along
    the rows)."""
    for spans, causal in (([(0, 13, 0, 5000)], True), ([(0, 3000, 0, 37)], False)):
        c = Case(ctx, dt, 5, 1, d, spans, causal, grad=True)
        c.forward()
        outs = c.grads()
        clean(ctx)
        c.check_forward()
        c.check_grads(outs)


@pytest.mark.parametrize("d", [72, 128])
def test_rows_on_16_bytes_alone(ctx, d):  # noqa: F811
    """Outputs whose rows begin on 16 bytes and not on 32, as columns of wider matrices."""
    c = Case(ctx, "bf16", 3, 1, d, packed(33, 1, 77), pad=8, grad=True)
    c.forward()
    outs = c.grads(pad=8)
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [1600, 3200, 4700, 6200, 7700, 9300])
def test_parts_of_several_counts(ctx, dt, n):  # noqa: F811
    """From 2 to 7 parts of a row of work, along the keys and along the rows."""
    for spans, causal in (([(0, 30, 0, n)], True), ([(0, n, 0, 30)], False)):
        c = Case(ctx, dt, 4, 1, 64, spans, causal, grad=True)
        c.forward()
        outs = c.grads()
        clean(ctx)
        c.check_forward()
        c.check_grads(outs)
