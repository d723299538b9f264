"""Rotary positions on the GPU (C ABI) against the fp64 oracle.

Tolerance: the angle is a fraction of a turn held to 2^-32 of one (1.5e-9 radians), its sine and cosine come from fp32 functions
good to 2 ulp of values up to 1 (2^-22), the rotation is two products and a sum (3 2^-24 of |a| + |b|), and the result is rounded
once to its type.
"""
import numpy as np
import pytest
import torch

import paper_2607_01125_gb300 as zo
from oracle import decoder

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 0.0, "bf16": 0.0, "fp16": 2.0 ** -25}
PARTS = dict(factor=8.0, low=1.0, high=4.0, original=8192)


@pytest.fixture(scope="module")
def ctx():
    c = zo.Context(0)
    yield c
    c.close()


def n64(t):
    return t.detach().double().cpu().numpy()


def rnd(seed, *shape, dt="fp32"):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(TYPES[dt])


def clean(ctx):
    torch.cuda.synchronize()
    assert ctx.device_status() == 0


def check(Y, X, pos, heads, head_dim, rot, base, layout, scaling, inverse, dt):
    x = n64(X).reshape(X.shape[0], heads, head_dim)
    f = decoder.frequencies(rot, base, scaling, **PARTS)
    want = decoder.rope(x, [int(p) for p in pos.cpu()], f, layout, inverse)
    turned = np.zeros(head_dim, dtype=bool)
    turned[:rot] = True
    h = rot // 2
    size = np.zeros_like(x)
    at = (slice(0, h), slice(h, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    size[..., at[0]] = size[..., at[1]] = np.abs(x[..., at[0]]) + np.abs(x[..., at[1]])
    got = n64(Y).reshape(x.shape)
    assert (got[..., rot:] == x[..., rot:]).all()
    # the oracle's own angle: positions up to 2^40 times frequencies with 2^-53
    far = max(1.0, float(pos.abs().max())) * 2.0 ** -51 if len(pos) else 0.0
    tol = size * (2.0 ** -22 + 3 * 2.0 ** -24 + 1.5e-9 + far) + UNIT[dt] * np.abs(want) * 1.01 + TINY[dt]
    err = np.abs(got - want)
    assert np.isfinite(got).all() and (err <= tol)[..., :rot].all(), float((err / np.maximum(tol, 1e-300)).max())


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,head_dim,rot,scaling", [(1, 1, 2, 2, "none"), (7, 3, 128, 128, "none"), (40, 5, 80, 32, "linear"),
                                                            (33, 2, 96, 48, "parts"), (5, 4, 10, 6, "base"), (300, 2, 256, 256, "parts"),
                                                            (64, 1, 21, 14, "none"), (11, 40, 128, 64, "base")])
def test_rope(ctx, dt, layout, rows, heads, head_dim, rot, scaling):
    X = rnd(rows + head_dim, rows, heads * head_dim, dt=dt)
    pos = torch.arange(rows, device=DEV) * 37 % 1000
    for inverse in (False, True):
        Y = torch.full_like(X, float("nan"))
        zo.zoact_rope_apply(ctx, X, pos, zo.rope(rot, base=500000.0, layout=layout, scaling=scaling, **PARTS), Y, heads, inverse)
        clean(ctx)
        check(Y, X, pos, heads, head_dim, rot, 500000.0, layout, scaling, inverse, dt)


@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("first", [0, -5, 1000000, 2 ** 31 - 20])
def test_rope_of_far_positions(ctx, idt, first):
    X = rnd(3, 17, 2 * 64)
    pos = torch.arange(first, first + 17, device=DEV, dtype=torch.int64).to(idt)
    Y = torch.empty_like(X)
    zo.zoact_rope_apply(ctx, X, pos, zo.rope(64), Y, 2)
    clean(ctx)
    check(Y, X, pos, 2, 64, 64, 10000.0, "half", "none", False, "fp32")


def test_rope_of_positions_beyond_32_bits(ctx):
    X = rnd(3, 5, 64)
    pos = 2 ** 33 + torch.arange(5, device=DEV) * 2 ** 32
    Y = torch.empty_like(X)
    zo.zoact_rope_apply(ctx, X, pos, zo.rope(64), Y, 1)
    clean(ctx)
    check(Y, X, pos, 1, 64, 64, 10000.0, "half", "none", False, "fp32")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt,pad,shift", [("bf16", 8, 0), ("bf16", 3, 0), ("fp16", 8, 1), ("fp32", 4, 2), ("fp32", 0, 4)])
def test_rope_of_column_views_and_in_place(ctx, layout, dt, pad, shift):
    """q and k columns of a wider output, blocks of one set of positions; rows that do and do not start on 16 bytes."""
    heads, d, T, nb = 3, 32, 13, 3
    full = rnd(9, nb * T, shift + heads * d + pad, dt=dt)
    X = full[:, shift:shift + heads * d]
    before = full.clone()
    pos = torch.arange(T, device=DEV, dtype=torch.int32) * 11
    r = zo.rope(32, layout=layout)
    Y = torch.empty(nb * T, heads * d, dtype=TYPES[dt], device=DEV)
    zo.zoact_rope_apply(ctx, X, pos, r, Y, heads)
    clean(ctx)
    assert torch.equal(full, before)
    check(Y, X, pos, heads, d, 32, 10000.0, layout, "none", False, dt)
    zo.zoact_rope_apply(ctx, X, pos, r, X, heads)
    clean(ctx)
    assert torch.equal(X, Y)
    assert torch.equal(full[:, :shift], before[:, :shift]) and torch.equal(full[:, shift + heads * d:], before[:, shift + heads * d:])


def test_rope_in_place_leaves_what_does_not_turn(ctx):
    X = rnd(4, 6, 2 * 40, dt="bf16")
    before = X.clone()
    zo.zoact_rope_apply(ctx, X, torch.arange(6, device=DEV), zo.rope(16), X, 2)
    clean(ctx)
    check(X, before, torch.arange(6, device=DEV), 2, 40, 16, 10000.0, "half", "none", False, "bf16")


def test_rope_captured(ctx):
    X, pos = rnd(4, 10, 64, dt="bf16"), torch.arange(10, device=DEV)
    Y, want = torch.empty_like(X), torch.empty_like(X)
    r = zo.rope(64)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.sync_stream()
        zo.zoact_rope_apply(ctx, X, pos, r, Y, 1)
    ctx.sync_stream()
    pos += 5
    graph.replay()
    zo.zoact_rope_apply(ctx, X, pos, r, want, 1)
    clean(ctx)
    assert torch.equal(Y, want)


def test_rope_of_nothing_and_refusals(ctx):
    r = zo.rope(16)
    zo.zoact_rope_apply(ctx, torch.empty(0, 32, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), r, torch.empty(0, 32, device=DEV), 2)
    clean(ctx)
    X, pos = rnd(1, 6, 32), torch.arange(6, device=DEV)
    Y = torch.empty_like(X)
    before = ctx.launch_count()
    bad = [lambda: zo.zoact_rope_apply(ctx, X, pos, r, Y, 3), lambda: zo.zoact_rope_apply(ctx, X, pos, r, Y, 4),      # heads, rot
           lambda: zo.zoact_rope_apply(ctx, X, pos[:4], r, Y, 2), lambda: zo.zoact_rope_apply(ctx, X, pos[:0], r, Y, 2),
           lambda: zo.zoact_rope_apply(ctx, X, pos.float(), r, Y, 2), lambda: zo.zoact_rope_apply(ctx, X, pos, r, Y[:5], 2),
           lambda: zo.zoact_rope_apply(ctx, X, pos, r, Y.half(), 2), lambda: zo.zoact_rope_apply(ctx, X, pos.cpu(), r, Y, 2),
           lambda: zo.zoact_rope_apply(ctx, X, pos, r, Y.t().contiguous().t(), 2), lambda: zo.zoact_rope_apply(ctx, X, pos, r, Y, 0)]
    for call in bad:
        with pytest.raises((ValueError, zo.ZoactError)):
            call()
    assert ctx.launch_count() == before
