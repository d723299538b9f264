"""Attention over packed sequences and its gradient on the GPU (C ABI) against the fp64 oracle.

Tolerances are bounds on the arithmetic.  F = 2^-24, u = half a step of a stored type.
  a score of D products in fp32 errs by (D + 4) F of its sum of magnitudes Z (the tensor core cuts its sums off: 2 F a step
    of 16, no more than that); the share of it, exp(s - m), by as much absolutely times its value, and by 2^-21 for the product by log2 e
    of scores and maxima below 64, the exponential (2 ulp) and the sums' scale;
  o: its shares rounded to the operands' type on the tensor cores (u, and below fp16's normal range 2^-25 of the largest share's
    unit), n terms summed in fp32 (n F, or 2 F for every 16 of them on the tensor cores), then one rounding (u);
  lse: the score's error, the sum's n F, and roundings of its own size (4 F).
The gradient's bounds are made alike by the oracle (oracle/decoder.py) for the O and lse that the forward call gave.
"""
import math

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
F = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = zo.Context(0)
    yield c
    c.close()


def n64(t):
    return t.detach().double().cpu().numpy()


def rnd(seed, *shape, std=1.0, dt="fp32"):
    return (torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) * std).to(TYPES[dt])


def clean(ctx):
    torch.cuda.synchronize()
    assert ctx.device_status() == 0


def plan_of(ctx, shape, spans, grad=False, idt=torch.int64):
    plan = torch.empty(zo.zoact_attention_plan_bytes(ctx, shape, grad=grad), dtype=torch.uint8, device=DEV)
    zo.zoact_attention_plan(ctx, shape, torch.tensor(spans, dtype=idt, device=DEV).view(-1, 4), plan, grad=grad)
    return plan


class Case:
    """Operands as columns of wider matrices (`pad` columns between rows), and outputs full of NaN."""

    def __init__(self, ctx, dt, heads, kv_heads, d, spans, causal=True, std=1.0, pad=0, rows_q=None, rows_k=None, seed=1, grad=False,
                 idt=torch.int64):
        self.ctx, self.dt, self.spans, self.causal = ctx, dt, [tuple(s) for s in spans], causal
        nq = max([s[0] + s[1] for s in spans], default=0) if rows_q is None else rows_q
        nk = max([s[2] + s[3] for s in spans], default=0) if rows_k is None else rows_k
        self.heads, self.kv_heads, self.d, self.nq, self.nk = heads, kv_heads, d, nq, nk
        self.scale = 1 / math.sqrt(d)

        def mat(i, rows, h, s=std):
            return rnd(seed * 10 + i, rows, h * d + pad, std=s, dt=dt)[:, :h * d]

        self.q, self.k, self.v = mat(1, nq, heads), mat(2, nk, kv_heads), mat(3, nk, kv_heads)
        self.dO = mat(4, nq, heads, 0.5)
        self.shape = zo.attention_shape(nq, nk, len(spans), heads, kv_heads, d, causal)
        self.plan = plan_of(ctx, self.shape, self.spans, grad, idt)
        self.O = torch.full((nq, heads * d + pad), float("nan"), dtype=TYPES[dt], device=DEV)[:, :heads * d]
        self.lse = torch.full((nq, heads), float("nan"), device=DEV)

    def h64(self, t, heads):
        return n64(t).reshape(t.shape[0], heads, self.d)

    def args64(self):
        return self.h64(self.q, self.heads), self.h64(self.k, self.kv_heads), self.h64(self.v, self.kv_heads)

    def forward(self):
        zo.zoact_attention(self.ctx, self.shape, self.plan, self.q, self.k, self.v, self.O, lse=self.lse)

    def check_forward(self):
        O, lse, A, Z, V = decoder.attention(*self.args64(), self.spans, self.causal, self.scale, size=True)
        n = max([s[3] for s in self.spans], default=0)
        u = UNIT[self.dt]
        es = (self.d + 4) * F * Z
        got, gl = self.h64(self.O, self.heads), n64(self.lse)
        none = np.isnan(lse)
        assert (np.isnan(gl) == none).all() and (np.isnan(got) == np.isnan(O)).all()      # rows of no sequence are left alone
        tol = (2 * es[..., None] + 2.0 ** -20 + (2 * n + 8) * F + u) * A + u * np.abs(O) * 1.01 + TINY[self.dt] * (1 + V)
        err = np.abs(got - O)
        assert (err[~none] <= tol[~none]).all(), float(np.nanmax(err / np.maximum(tol, 1e-300)))
        empty = lse == -np.inf
        assert (gl[empty] == -np.inf).all()
        some = ~none & ~empty
        lt = es + 2.0 ** -20 + (n + 8) * F + 4 * F * np.abs(np.where(some, lse, 0))
        assert (np.abs(gl[some] - lse[some]) <= lt[some]).all()

    def grads(self, pad=0):
        outs = []
        for rows, h in ((self.nq, self.heads), (self.nk, self.kv_heads), (self.nk, self.kv_heads)):
            outs.append(torch.full((rows, h * self.d + pad), float("nan"), dtype=TYPES[self.dt], device=DEV)[:, :h * self.d])
        zo.zoact_attention_grad(self.ctx, self.shape, self.plan, self.dO, self.q, self.k, self.v, self.O, self.lse, *outs)
        return outs

    def check_grads(self, outs):
        n = max([max(s[1] * self.heads // self.kv_heads, s[3]) for s in self.spans], default=0)
        # below 2^-126 fp32 has no (or few) digits left: a share, and what is made of it, is off by that much whatever its size
        u, tiny = UNIT[self.dt], max(TINY[self.dt], 2.0 ** -126)
        lse = n64(self.lse)
        top = np.abs(lse[np.isfinite(lse)]).max(initial=0.0)
        error = (2.0 ** -20 + 4 * F * top, (self.d + 4) * F, (self.d + 4) * F, u, 64 * tiny, (2 * n + 8) * F)
        q, k, v = self.args64()
        res = decoder.attention_grad(self.h64(self.dO, self.heads), q, k, v, self.h64(self.O, self.heads), lse, self.spans,
                                     self.causal, self.scale, error)
        for name, got, want, tol, h in zip(("dq", "dk", "dv"), outs, res[:3], res[3:], (self.heads, self.kv_heads, self.kv_heads)):
            g = self.h64(got, h)
            assert (np.isnan(g) == np.isnan(want)).all(), name
            at = ~np.isnan(want)
            t = tol + u * np.abs(want) * 1.01 + tiny
            err = np.abs(g - want)
            worst = np.unravel_index(np.argmax(np.where(at, err / np.maximum(t, 1e-300), 0.0)), err.shape)
            assert (err[at] <= t[at]).all(), (name, worst, g[worst], want[worst], t[worst], float((err[at] / np.maximum(t[at], 1e-300)).max()))


def packed(*lens):
    return [tuple(r) for r in zo.attention_spans(lens).tolist()]


SHAPES = [(4, 4, 128), (8, 2, 128), (5, 1, 64), (2, 2, 80), (6, 2, 24), (2, 1, 33), (3, 3, 192)]


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_packed_sequences(ctx, dt, heads, kv_heads, d, causal):
    c = Case(ctx, dt, heads, kv_heads, d, packed(1, 2, 0, 63, 64, 65, 130, 200), causal)
    c.forward()
    clean(ctx)
    c.check_forward()


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_gradient_of_packed_sequences(ctx, dt, heads, kv_heads, d, causal):
    c = Case(ctx, dt, heads, kv_heads, d, packed(1, 2, 0, 63, 64, 65, 130, 200), causal, grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)
    again = c.grads()
    clean(ctx)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))          # the same bits


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 2), (16, 1)])
@pytest.mark.parametrize("n", [1, 127, 128, 129, 255, 256, 257, 511, 1000])
def test_lengths_around_the_tiles(ctx, dt, heads, kv_heads, n):
    c = Case(ctx, dt, heads, kv_heads, 64, packed(n), grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,d", [(8, 2, 128), (4, 4, 64), (8, 1, 128), (2, 2, 40)])
@pytest.mark.parametrize("queries", [1, 3, 40])
def test_new_tokens_against_a_cache(ctx, dt, heads, kv_heads, d, queries):
    """Queries behind keys that lie in slots with room (NaN there), one slot shared, keys up to those that are cut in parts."""
    keys = [queries, 64, 129, 700, 3000, 700]
    slots = [0, 100, 300, 500, 1500, 500]
    spans = [(i * (queries + 1), queries, s, max(n, queries)) for i, (n, s) in enumerate(zip(keys, slots))]
    c = Case(ctx, dt, heads, kv_heads, d, spans, rows_q=6 * (queries + 1), rows_k=5000)
    used = torch.zeros(5000, dtype=torch.bool, device=DEV)
    for _, _, s, n in spans:
        used[s:s + n] = True
    c.k[~used] = float("nan")
    c.v[~used] = float("nan")
    c.q[queries::queries + 1] = float("nan")
    c.forward()
    clean(ctx)
    assert torch.isfinite(c.lse[:queries]).all()
    keep = c.k.clone(), c.v.clone(), c.q.clone()
    c.k, c.v, c.q = (torch.nan_to_num(t) for t in keep)
    c.check_forward()


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
def test_rows_that_see_no_key(ctx, dt):
    """More queries than keys, no keys at all, keys without a query."""
    spans = [(0, 10, 0, 3), (10, 150, 3, 20), (160, 7, 23, 0), (167, 0, 23, 40), (167, 2, 63, 2)]
    c = Case(ctx, dt, 4, 2, 64, spans, grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)
    assert (outs[1][23:63] == 0).all() and (outs[2][23:63] == 0).all() and (outs[0][160:167] == 0).all()


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_lies_outside_a_sequence_does_not_reach_it(ctx, dt, bad):
    spans = [(3, 70, 5, 70), (100, 33, 80, 140), (140, 1, 300, 9)]
    c = Case(ctx, dt, 4, 2, 64, spans, grad=True, rows_q=160, rows_k=330)
    for t, col in ((c.q, 0), (c.dO, 0), (c.k, 2), (c.v, 2)):
        inside = torch.zeros(t.shape[0], dtype=torch.bool, device=DEV)
        for s in spans:
            inside[s[col]:s[col] + s[col + 1]] = True
        t[~inside] = bad
    c.forward()
    c.O[torch.isnan(c.lse[:, 0])] = bad
    outs = c.grads()
    clean(ctx)
    at_q, at_k = torch.zeros(160, dtype=torch.bool), torch.zeros(330, dtype=torch.bool)
    for s in spans:
        at_q[s[0]:s[0] + s[1]] = True
        at_k[s[2]:s[2] + s[3]] = True
    for t, at in ((outs[0], at_q), (outs[1], at_k), (outs[2], at_k), (c.lse, at_q)):
        assert torch.isfinite(t.cpu()[at]).all() and torch.isnan(t.cpu()[~at]).all()
    for name in ("q", "k", "v", "dO"):
        setattr(c, name, torch.nan_to_num(getattr(c, name), posinf=0.0, neginf=0.0))
    c.O = torch.where(torch.isnan(c.lse[:, :1]), torch.full_like(c.O, float("nan")), c.O)
    c.check_forward()
    c.O = torch.nan_to_num(c.O)
    c.check_grads(outs)


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
def test_a_sequence_with_nan_leaves_the_others(ctx, dt):
    c = Case(ctx, dt, 4, 2, 64, packed(50, 60, 70), grad=True)
    c.k[60], c.v[75], c.q[70], c.dO[90] = (float("nan") for _ in range(4))
    c.forward()
    outs = c.grads()
    torch.cuda.synchronize()
    for t in (c.O, c.lse, *outs):
        assert torch.isfinite(t[:50]).all() and torch.isfinite(t[110:]).all()
        assert torch.isnan(t[50:110]).any()


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
def test_large_scores(ctx, dt):
    """Scores of hundreds: the running maximum moves often, and most shares vanish."""
    c = Case(ctx, dt, 4, 2, 64, packed(300, 33), std=6.0, grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("rising", [True, False])
def test_scores_that_rise_along_the_keys(ctx, dt, rising):
    """Every block of keys above (or below) the last: a maximum that is raised at each step, or never."""
    c = Case(ctx, dt, 2, 1, 64, [(0, 300, 0, 1200)])
    ramp = torch.linspace(0, 40, 1200, device=DEV)[:, None] * (1 if rising else -1)
    c.q[:], c.k[:] = 1.0, (ramp / 8 + 0.01 * rnd(5, 1200, 64)).to(TYPES[dt])
    c.forward()
    clean(ctx)
    c.check_forward()


@pytest.mark.parametrize("dt,pad", [("bf16", 8), ("bf16", 3), ("fp16", 1), ("fp32", 3), ("fp16", 16)])
def test_columns_of_wider_outputs(ctx, dt, pad):
    c = Case(ctx, dt, 4, 2, 64, packed(70, 129), pad=pad, grad=True)
    c.forward()
    outs = c.grads(pad)
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)
    base = c.O._base if c.O._base is not None else c.O
    assert torch.isnan(base[:, 4 * 64:]).all()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
def test_long_rows_of_work_are_cut_and_joined(ctx, dt, idt):
    """Few rows of work, long in keys (forward, dq) and in queries (dk, dv): parts, joined in order, twice the same bits."""
    c = Case(ctx, dt, 2, 1, 64, [(0, 130, 0, 5000)], causal=True, grad=True, idt=idt)
    c.forward()
    outs = c.grads()
    first = c.O.clone(), c.lse.clone()
    c.forward()
    again = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)
    assert torch.equal(c.O, first[0]) and torch.equal(c.lse, first[1]) and all(torch.equal(a, b) for a, b in zip(outs, again))
    c = Case(ctx, dt, 4, 1, 64, [(0, 2000, 0, 100)], causal=False, grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)


@pytest.mark.parametrize("dt,heads,kv_heads", [("bf16", 8, 8), ("fp32", 4, 4)])
def test_rows_behind_32_bits(ctx, dt, heads, kv_heads):
    """A cache of more than 2^31 elements (fp32: 2^31 bytes), its last rows used, and rows of q as far apart."""
    d = 128 if dt == "bf16" else 64
    rows = 2 ** 31 // (kv_heads * d) + 1000 if dt == "bf16" else 2 ** 29 // (kv_heads * d) * 2 + 1000
    cache = [torch.empty(rows, kv_heads * d, dtype=TYPES[dt], device=DEV) for _ in range(2)]
    n, first = 300, rows - 310
    spans = [(0, 2, first, n)]
    small = Case(ctx, dt, heads, kv_heads, d, [(0, 2, 0, n)])
    for t, x in zip(cache, (small.k, small.v)):
        t[first:first + n] = x
    shape = zo.attention_shape(2, rows, 1, heads, kv_heads, d)
    plan = plan_of(ctx, shape, spans)
    wide = torch.empty(2, 2 ** 31 // 2 + 64, dtype=TYPES[dt], device=DEV)
    q = wide[:, :heads * d]
    q.copy_(small.q)
    zo.zoact_attention(ctx, shape, plan, q, cache[0], cache[1], small.O, lse=small.lse)
    clean(ctx)
    small.check_forward()


@pytest.mark.parametrize("power", [0, 6, 12])
def test_small_gradients_in_fp16(ctx, power):
    """Powers of two of dO pass through: what is rounded to fp16 on the way is scaled to dO's size, so that a small dO loses
    nothing but the last roundings below fp16's normal range."""
    c = Case(ctx, "fp16", 4, 2, 64, packed(300, 40), grad=True)
    c.forward()
    small = c.dO.float() * 2.0 ** -power
    c.dO.copy_(torch.where(small.abs() < 2.0 ** -14, torch.zeros_like(small), small))       # exact
    part = c.grads()
    c.dO.mul_(2.0 ** power)
    full = c.grads()
    clean(ctx)
    for a, b in zip(full, part):
        a, b = n64(a), n64(b) * 2.0 ** power
        assert (np.abs(a - b) <= 2.0 ** -11 * np.abs(a) + 2.0 ** -24 * 2.0 ** power).all()


@pytest.mark.parametrize("dO,v", [(2.0 ** -6, 256.0), (2.0 ** -20, 30000.0), (60.0, 2.0 ** -12), (1.0, 0.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_large_and_small_values_in_fp16(ctx, dO, v, d):
    """dO and v of one sign pattern: dP and dS are as large as they can be for their sizes, and the gradients fit."""
    c = Case(ctx, "fp16", 4, 2, d, packed(200, 40), grad=True, std=0.5)
    signs = (torch.arange(d, device=DEV) % 3 - 1).half()
    c.dO.copy_(dO * signs.repeat(4) * (0.5 + rnd(5, c.nq, 1).sigmoid().half()))
    c.v.copy_(v * signs.repeat(2) * rnd(6, c.nk, 1).sign().half())
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_grads(outs)


def test_a_call_leaves_nothing_to_the_next(ctx):
    """fp16: large values, then small ones with the same plan, give what a fresh plan gives; the forward call's plan too."""
    got = []
    for before in (False, True):
        c = Case(ctx, "fp16", 4, 2, 64, packed(300, 40), grad=True)
        c.forward()
        small = c.dO * 2.0 ** -8
        if before:
            c.dO.mul_(100)
            c.v.mul_(64)
            c.forward()
            c.grads()
            c.v.div_(64)
            c.forward()
        c.dO.copy_(small)
        got.append(c.grads())
        clean(ctx)
    v = Case(ctx, "fp16", 4, 2, 64, packed(300, 40)).v
    assert torch.equal(v, c.v)                    # times 64 and back is exact
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_large_values_outside_of_the_sequences_cost_small_gradients_nothing(ctx):
    """fp16: the scale of dS comes from the sequences' rows alone."""
    spans = [(7, 60, 7, 60), (80, 50, 80, 50)]
    got = []
    for outside in (0.0, 60000.0, float("inf"), float("nan")):
        c = Case(ctx, "fp16", 4, 2, 64, spans, grad=True, rows_q=140, rows_k=140)
        c.dO.mul_(2.0 ** -10)
        inside = torch.zeros(140, dtype=torch.bool, device=DEV)
        inside[7:67] = inside[80:130] = True
        c.dO[~inside] = c.v[~inside] = outside
        c.forward()
        c.O[~inside] = outside
        outs = c.grads()
        clean(ctx)
        got.append([t[inside].clone() for t in outs])
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(other, got[0]))


def test_many_short_sequences(ctx):
    rng = np.random.default_rng(3)
    c = Case(ctx, "bf16", 4, 2, 64, packed(*rng.integers(0, 6, 3000)), grad=True)
    c.forward()
    outs = c.grads()
    clean(ctx)
    c.check_forward()
    c.check_grads(outs)


def test_wide_groups(ctx):
    for heads in (48, 71, 128):
        c = Case(ctx, "bf16", heads, 1, 64, packed(5, 40), grad=True)
        c.forward()
        outs = c.grads()
        clean(ctx)
        c.check_forward()
        c.check_grads(outs)


def test_nothing_to_do(ctx):
    for spans in ([], packed(0, 0)):
        c = Case(ctx, "bf16", 4, 2, 64, spans, grad=True, rows_q=9, rows_k=9)
        c.forward()
        outs = c.grads()
        clean(ctx)
        assert all(torch.isnan(t).all() for t in (c.O, c.lse, *outs))
    c = Case(ctx, "bf16", 4, 2, 64, [], grad=True, rows_q=0, rows_k=0)
    c.forward()
    c.grads()
    clean(ctx)


def test_without_log_sum_exps_and_another_scale(ctx):
    c = Case(ctx, "bf16", 4, 2, 64, packed(100))
    c.forward()
    O = torch.empty_like(c.O)
    zo.zoact_attention(ctx, c.shape, c.plan, c.q, c.k, c.v, O)
    clean(ctx)
    assert torch.equal(O, c.O)
    c.scale = 0.3
    zo.zoact_attention(ctx, c.shape, c.plan, c.q, c.k, c.v, c.O, lse=c.lse, scale=0.3)
    clean(ctx)
    c.check_forward()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_captured_and_replayed_with_other_spans(ctx, dt):
    a, b = packed(40, 0, 90), packed(30, 70, 30)
    c = Case(ctx, dt, 4, 2, 64, a, grad=True)
    c.forward()
    outs = c.grads()                                     # scratch before the capture
    spans = torch.tensor(a, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        ctx.sync_stream()
        zo.zoact_attention_plan(ctx, c.shape, spans, c.plan, grad=True)
        c.forward()
        zo.zoact_attention_grad(ctx, c.shape, c.plan, c.dO, c.q, c.k, c.v, c.O, c.lse, *outs)
    ctx.sync_stream()
    for s in (b, a):
        spans.copy_(torch.tensor(s, device=DEV))
        graph.replay()
        clean(ctx)
        c.spans = s
        c.check_forward()
        c.check_grads(outs)


def test_bad_spans_and_plans_write_nothing(ctx):
    good = packed(10, 20)
    bad = [[(0, 10, 0, 10), (9, 20, 10, 20)], [(0, 10, 0, 10), (10, 21, 10, 20)], [(0, 10, 0, 31), (10, 20, 10, 20)],
           [(-1, 10, 0, 10), (10, 20, 10, 20)], [(0, -1, 0, 10), (10, 20, 10, 20)], [(0, 10, 0, 2 ** 62), (10, 20, 10, 20)],
           [(2 ** 63 - 1, 2, 0, 10), (10, 20, 10, 20)], [(10, 20, 10, 20), (0, 10, 0, 10)]]
    for grad in (False, True):
        for spans in bad + ([[(0, 10, 5, 20), (10, 20, 10, 20)]] if grad else []):
            c = Case(ctx, "bf16", 4, 2, 64, good, grad=grad)
            plan_of(ctx, c.shape, spans, grad)
            c.plan = plan_of(ctx, c.shape, spans, grad)
            c.forward()
            outs = c.grads() if grad else []
            torch.cuda.synchronize()
            assert ctx.device_status() == -1
            assert all(torch.isnan(t).all() for t in (c.O, c.lse, *outs))
    # a plan of another shape, one without the gradient's lists (in room for them), and none at all
    c = Case(ctx, "bf16", 4, 2, 64, good)
    other = Case(ctx, "bf16", 4, 4, 64, good, grad=True)
    room = torch.zeros(zo.zoact_attention_plan_bytes(ctx, c.shape, grad=True), dtype=torch.uint8, device=DEV)
    for plan, grad in ((other.plan, False), (room, False), (room, True), (torch.cat([c.plan, room])[:room.numel()], True)):
        d = Case(ctx, "bf16", 4, 2, 64, good)
        d.plan = plan.clone()
        d.lse.zero_()
        if grad:
            outs = d.grads()
        else:
            d.forward()
            outs = [d.O]
        torch.cuda.synchronize()
        assert ctx.device_status() == -1
        assert all(torch.isnan(t).all() for t in outs)
    clean(ctx)


def test_refusals(ctx):
    c = Case(ctx, "bf16", 4, 2, 64, packed(10), grad=True)
    f = dict(lse=c.lse)
    before = ctx.launch_count()
    A, G = zo.zoact_attention, zo.zoact_attention_grad
    p, s = c.plan, c.shape
    calls = [lambda: A(ctx, s, p, c.q[:9], c.k, c.v, c.O, **f), lambda: A(ctx, s, p, c.q, c.k.float(), c.v, c.O, **f),
             lambda: A(ctx, s, p, c.q, c.k, c.v[:, :64], c.O, **f), lambda: A(ctx, s, p, c.q, c.k, c.v, c.O, lse=c.lse[:, :2]),
             lambda: A(ctx, s, p, c.q, c.k, c.v, c.O, scale=0.0), lambda: A(ctx, s, p, c.q, c.k, c.v, c.O, scale=float("nan")),
             lambda: A(ctx, s, p, c.q, c.k, c.v, c.O, scale=-1.0), lambda: A(ctx, s, p, c.q.cpu(), c.k, c.v, c.O),
             lambda: A(ctx, s, p[:100], c.q, c.k, c.v, c.O), lambda: A(ctx, s, p.float(), c.q, c.k, c.v, c.O),
             lambda: A(ctx, s, p, c.q.t().contiguous().t(), c.k, c.v, c.O),
             lambda: G(ctx, s, p, c.dO, c.q, c.k, c.v, c.O, None, c.q, c.k, c.v),
             lambda: G(ctx, s, p, c.dO, c.q, c.k, c.v, c.O, c.lse, c.q.float(), c.k, c.v),
             lambda: G(ctx, s, plan_small, c.dO, c.q, c.k, c.v, c.O, c.lse, c.q, c.k, c.v),
             lambda: zo.zoact_attention_plan(ctx, s, torch.zeros(2, 4, dtype=torch.int64, device=DEV), p),
             lambda: zo.zoact_attention_plan(ctx, s, torch.zeros(1, 4, device=DEV), p),
             lambda: zo.zoact_attention_plan(ctx, s, torch.zeros(1, 4, dtype=torch.int64), p)]
    plan_small = torch.empty(zo.zoact_attention_plan_bytes(ctx, s), dtype=torch.uint8, device=DEV)
    for i, call in enumerate(calls):
        with pytest.raises((ValueError, zo.ZoactError)):
            call()
            raise AssertionError(i)
    for shape in ((1, 1, 1, 3, 2, 64), (1, 1, 1, 129, 1, 64), (1, 1, 1, 1, 1, 257), (-1, 1, 1, 1, 1, 8), (1, 1, 1, 0, 1, 8),
                  (2 ** 31 - 100, 1, 1, 1, 1, 8), (1, 2 ** 31 - 100, 1, 1, 1, 8), (2 ** 27, 1, 1, 65536, 65536, 8)):
        with pytest.raises(ValueError):
            zo.zoact_attention_plan_bytes(ctx, zo.attention_shape(*shape))
    # log-sum-exps that begin inside of an element
    st = zo.load().zoact_attention(ctx.handle, s, p.data_ptr(), c.q.data_ptr(), 256, c.k.data_ptr(), 128, c.v.data_ptr(), 128, 1, 0.125,
                                   c.O.data_ptr(), 256, c.lse.data_ptr() + 2)
    assert st == -1
    assert ctx.launch_count() == before
    clean(ctx)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_rotation_attention_and_back_as_one_path(ctx, dt):
    """q/k/v in one buffer, q and k turned in place in both blocks, attention, and the gradient back through both, against the
    oracle's gradient of the same chain and against differences of its loss."""
    heads, kv, d, T, nb = 4, 2, 64, 50, 2
    qkv = rnd(1, nb * T, (heads + 2 * kv) * d, dt=dt)
    start = qkv.clone()
    pos = torch.cat([torch.arange(20), torch.arange(30)]).to(DEV)
    r = zo.rope(48)
    spans = [tuple(x) for x in zo.attention_spans([20, 30] * nb).tolist()]
    turned = qkv[:, :(heads + kv) * d]
    zo.zoact_rope_apply(ctx, turned, pos, r, turned, heads + kv)
    q, k, v = qkv[:, :heads * d], qkv[:, heads * d:(heads + kv) * d], qkv[:, (heads + kv) * d:]
    shape = zo.attention_shape(nb * T, nb * T, len(spans), heads, kv, d)
    plan = plan_of(ctx, shape, spans, True)
    O, lse = torch.empty(nb * T, heads * d, dtype=TYPES[dt], device=DEV), torch.empty(nb * T, heads, device=DEV)
    dO = rnd(2, nb * T, heads * d, dt=dt)
    zo.zoact_attention(ctx, shape, plan, q, k, v, O, lse=lse)
    grad = torch.empty_like(qkv)
    zo.zoact_attention_grad(ctx, shape, plan, dO, q, k, v, O, lse, grad[:, :heads * d], grad[:, heads * d:(heads + kv) * d],
                            grad[:, (heads + kv) * d:])
    back = grad[:, :(heads + kv) * d]
    zo.zoact_rope_apply(ctx, back, pos, r, back, heads + kv, inverse=True)
    clean(ctx)

    f, P = decoder.frequencies(48, 10000.0), [int(x) for x in pos]
    x0 = n64(start).reshape(nb * T, heads + 2 * kv, d)
    G = n64(dO).reshape(nb * T, heads, d)

    def chain(x):
        y = np.concatenate([decoder.rope(x[:, :heads + kv], P, f, "half"), x[:, heads + kv:]], axis=1)
        return y[:, :heads], y[:, heads:heads + kv], y[:, heads + kv:]

    y = chain(x0)
    o, l = decoder.attention(*y, spans, True, d ** -0.5)
    want = np.concatenate(decoder.attention_grad(G, *y, o, l, spans, True, d ** -0.5), axis=1)
    want[:, :heads + kv] = decoder.rope(want[:, :heads + kv], P, f, "half", inverse=True)
    rng = np.random.default_rng(4)
    for _ in range(6):
        step = rng.standard_normal(x0.shape)
        up, down = (np.sum(decoder.attention(*chain(x0 + e * step), spans, True, d ** -0.5)[0] * G) for e in (1e-6, -1e-6))
        assert abs((up - down) / 2e-6 - (want * step).sum()) <= 1e-6 * np.abs(want * step).sum()
    # two roundings of each operand and of O before, of the shares within, and of the gradient after: a few units of the rows' size
    got, u = n64(grad).reshape(want.shape), UNIT[dt]
    size = np.sqrt((want ** 2).mean())
    assert np.sqrt(((got - want) ** 2).mean()) <= (4 * u + 1e-5) * size
    assert np.abs(n64(O).reshape(o.shape) - o).max() <= (8 * u + 1e-5) * np.abs(x0).max()
