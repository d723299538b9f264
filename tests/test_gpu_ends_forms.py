"""The forms of the kernels at a language model's ends that large calls take, against their formulas in fp64 on the GPU: cross
entropy with the rows on the MMA's M side and direct stores of the head's gradient, layer norm with two rows a block and
a ring that goes round, tokens sorted in one to three passes, and all of them in a captured graph.

Tolerances are bounds on the arithmetic, per element: F = 2^-24; a sum of k terms in fp32 errs by at most k F times the sum of
their magnitudes, G is rounded to the operands' type (bf16 2^-8, fp16 2^-11; fp32: three parts, 2^-21), its kept logits
to 2^-12, and every result once to its own type (fp16 below its normal range: by 2^-25).
"""
import pytest
import torch

import paper_2607_01125_gb300 as zo

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


def rnd(seed, *shape, std=1.0, dt="fp32"):
    g = torch.Generator(DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(TYPES[dt])


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def nans(*shape, dt="fp32"):
    return torch.full(shape, float("nan"), dtype=TYPES[dt], device=DEV)


def clean(ctx):
    torch.cuda.synchronize()
    assert ctx.device_status() == 0


def within(got, want, tol):
    got = got.double()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert (over <= 0).all(), float(((got - want).abs() / torch.as_tensor(tol, device=DEV).clamp(min=1e-300)).max())


# ---- cross entropy ----
def _ce_reference(H, W, t, nb):
    """Logits' error bounds, the shares P, losses and log-sum-exps in fp64, rows on the first axis."""
    h, w, tt = H.double(), W.double(), t.repeat(nb)
    z = h @ w.t()
    lse = torch.logsumexp(z, dim=1)
    ez = (H.shape[1] + 8) * F * (h.abs() @ w.abs().t())
    zt = z.gather(1, tt.clamp(min=0)[:, None])[:, 0]
    loss = torch.where(tt >= 0, lse - zt, torch.zeros_like(lse))
    return h, w, ez, torch.exp(z - lse[:, None]), loss, lse


# rows on the M side, by the rule on 152 SMs (the first two fp32 cases: on the N side); two, three, one and many groups of K; both dimensions ragged; the head's gradient
# through shared memory (up to 13 K-blocks of 64 rows) and from registers
@pytest.mark.parametrize("dt,T,d,vocab", [("bf16", 601, 520, 20011), ("fp16", 601, 520, 20011), ("bf16", 1003, 1032, 20011),
                                          ("fp16", 1003, 1032, 20011), ("bf16", 4095, 264, 1009), ("fp16", 4095, 264, 1009),
                                          ("fp32", 1003, 260, 5003), ("fp32", 601, 1028, 1009), ("fp32", 1021, 260, 20011)])
def test_cross_entropy_of_many_rows(ctx, dt, T, d, vocab):
    W = rnd(2, vocab, d, std=2.0 / d ** 0.5, dt=dt)
    t = torch.randint(0, vocab, (T,), generator=gen(3), device=DEV)
    t[torch.rand(T, generator=gen(4), device=DEV) < 0.15] = -100
    N = int((t >= 0).sum())
    H2 = torch.cat([rnd(1, T, d, dt=dt), rnd(5, T, d, dt=dt)])
    h, w, ez, P, wloss, wlse = _ce_reference(H2, W, t, 2)
    el = 2 * ez.max(dim=1).values + 2.0 ** -20 + 4 * F * wlse.abs()
    loss, lse, mean = nans(2 * T), nans(2 * T), torch.full((2,), float("nan"), dtype=torch.float64, device=DEV)
    zo.zoact_ce_loss(ctx, H2, W, t, n_blocks=2, loss=loss, lse=lse, mean=mean)
    clean(ctx)
    within(lse, wlse, el)
    within(loss, wloss, el + F * wloss.abs())
    within(mean, wloss.view(2, T).sum(dim=1) / N, float(el.max()))
    one, one_mean = nans(T), torch.empty(1, dtype=torch.float64, device=DEV)
    zo.zoact_ce_loss(ctx, H2[:T], W, t, loss=one, mean=one_mean)
    clean(ctx)
    within(one, wloss[:T], el[:T] + F * wloss[:T].abs())
    del H2

    h, ez, P = h[:T], ez[:T], P[:T]
    H = h.to(TYPES[dt])
    counted = (t >= 0)[:, None]
    P = P * counted
    G = P.clone()
    G[torch.arange(T, device=DEV), t.clamp(min=0)] -= counted[:, 0].double()
    ug = 2.0 ** -21 if dt == "fp32" else 1.01 * UNIT[dt] + 2.0 ** -11
    eg = ug * G.abs() + (ez + ez.max(dim=1, keepdim=True).values + 2.0 ** -20) * P
    eg += (0 if dt == "fp32" else 2.0 ** -25) * counted
    scale = 3.0 / N
    wh, ww = scale * (G @ w), scale * (G.t() @ h)
    th = scale * (eg @ w.abs() + (vocab + 8) * F * (G.abs() @ w.abs()))
    tw = scale * (eg.t() @ h.abs() + (T + 8) * F * (G.abs().t() @ h.abs()))
    for wt in {dt, "fp32"}:
        dH, dW, loss2, lse2 = nans(T, d, dt=dt), nans(vocab, d, dt=wt), nans(T), nans(T)
        zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=dW, loss=loss2, lse=lse2, mean=one_mean, grad_scale=3.0)
        clean(ctx)
        within(lse2, wlse[:T], el[:T])
        assert torch.equal(loss2, one)
        within(dH, wh, th + UNIT[dt] * (wh.abs() + th) + TINY[dt])
        within(dW, ww, tw + UNIT[wt] * (ww.abs() + tw) + TINY[wt])
        assert (dH[t < 0] == 0).all()
        again = nans(vocab, d, dt=wt)
        zo.zoact_ce_grad(ctx, H, W, t, dW=again, grad_scale=3.0)
        clean(ctx)
        assert torch.equal(again, dW)
        if wt == "fp32":
            zo.zoact_ce_grad(ctx, H, W, t, dW=again, grad_scale=3.0, accumulate=True)
            clean(ctx)
            within(again, 2 * ww, 2 * tw + 4 * F * ww.abs())


# ---- layer norm ----
def _depth(n):
    return n / 32 + 16                                   # terms in a row on one thread, and the joins


def _norm(ctx, X, g, b, dt, eps=1e-5):
    rows, n = X.shape
    Y, mean, rstd = nans(rows, n, dt=dt), nans(rows), nans(rows)
    zo.zoact_layer_norm(ctx, X, g, b, Y, eps=eps, mean=mean, rstd=rstd)
    clean(ctx)
    x, gg, bb = X.double(), g.double(), b.double()
    wm = x.mean(dim=1)
    ws = ((x - wm[:, None]).square().mean(dim=1) + float(torch.tensor(eps))).rsqrt()
    k = _depth(n)
    em = k * F * x.abs().mean(dim=1) + F * wm.abs()
    es = (2 * k + 8) * F + (ws * em) ** 2
    within(mean, wm, em)
    within(rstd, ws, es * ws)
    wy = (x - wm[:, None]) * ws[:, None] * gg + bb
    xh = (x - wm[:, None]).abs() * ws[:, None]
    ty = gg.abs() * (ws[:, None] * em[:, None] + xh * (es[:, None] + 3 * F)) + 2 * F * (wy.abs() + bb.abs())
    within(Y, wy, ty + UNIT[dt] * (wy.abs() + ty) + TINY[dt])


@pytest.mark.parametrize("dt,pt", [("fp32", "fp32"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("times,n", [(4, 256), (8, 256), (4, 512), (8, 1032), (4, 4096), (5, 5120)])
def test_layer_norm_of_many_rows(ctx, dt, pt, times, n):
    """From four rows an SM on two of them share a block (of one warp each, of several; one vector a thread and two); an odd number
    of rows, whose last block has one."""
    rows = times * ctx.sm_count() + 1
    X = (rnd(1, rows, n) * torch.exp(rnd(2, rows, 1)) + 3 * rnd(3, rows, 1)).to(TYPES[dt])
    _norm(ctx, X, (1 + 0.3 * rnd(4, n)).to(TYPES[pt]), rnd(5, n, dt=pt), dt)


# A ring has at most 8 stages, and a block keeps the statistics of 32 rows at a time.  Blocks on an SM by width: 8 at 64,
# 2 (16 bits) or 1 at 4096, 1 at 8192 and at 7680 in fp32 (4 vectors a thread).
@pytest.mark.parametrize("dt,per_sm,rounds,n", [("bf16", 8, 67, 64), ("fp32", 8, 67, 64), ("fp16", 2, 12, 4096), ("fp32", 1, 12, 4096),
                                                ("bf16", 1, 35, 8192), ("fp32", 1, 9, 7680)])
def test_layer_norm_gradient_of_a_ring_that_goes_round(ctx, dt, per_sm, rounds, n):
    rows = rounds * per_sm * ctx.sm_count() + 5
    X, dY = rnd(1, rows, n, dt=dt), rnd(2, rows, n, dt=dt)
    g = 1 + 0.3 * rnd(3, n)
    mean, rstd = 0.1 * rnd(4, rows), torch.exp(0.3 * rnd(5, rows))
    dX, dg, db = nans(rows, n, dt=dt), nans(n), nans(n)
    zo.zoact_layer_norm_grad(ctx, dY, X, g, mean, rstd, dX=dX, dgain=dg, dbias=db)
    clean(ctx)
    s = rstd.double()[:, None]
    xh, dy = (X.double() - mean.double()[:, None]) * s, dY.double()
    within(dg, (dy * xh).sum(dim=0), (rows + 8) * F * (dy * xh).abs().sum(dim=0))
    within(db, dy.sum(dim=0), (rows + 8) * F * dy.abs().sum(dim=0))
    u = dy * g.double()
    tol = (_depth(n) + 8) * F * (u.abs().mean(dim=1, keepdim=True) + xh.abs() * (u * xh).abs().mean(dim=1, keepdim=True))
    tol = s * (tol + 8 * F * u.abs())
    want = s * (u - u.mean(dim=1, keepdim=True) - xh * (u * xh).mean(dim=1, keepdim=True))
    within(dX, want, tol + UNIT[dt] * (want.abs() + tol) + TINY[dt])
    dX1, dg1 = torch.empty_like(dX), torch.empty_like(dg)
    zo.zoact_layer_norm_grad(ctx, dY, X, g, mean, rstd, dX=dX1, dgain=dg1)
    clean(ctx)
    assert torch.equal(dX, dX1) and torch.equal(dg, dg1)


# ---- embedding gradient ----
def _embed_grad(ctx, ids, vocab, d, dt, accumulate, status=0):
    n = len(ids)
    dY, start = rnd(2, n, d, dt=dt), rnd(3, vocab, d)
    dE = start.clone() if accumulate else nans(vocab, d)
    zo.zoact_embed_grad(ctx, dY, ids, dE, scale=0.75, accumulate=accumulate)
    torch.cuda.synchronize()
    assert ctx.device_status() == status
    real = (ids >= 0) & (ids < vocab)
    want = start.double() if accumulate else torch.zeros(vocab, d, dtype=torch.float64, device=DEV)
    size, count = want.abs(), torch.bincount(ids[real].long(), minlength=vocab)[:, None]
    want.index_add_(0, ids[real].long(), 0.75 * dY.double()[real])
    size.index_add_(0, ids[real].long(), 0.75 * dY.double()[real].abs())
    within(dE, want, (count + 3) * F * size + F * want.abs())
    if accumulate:
        none = count[:, 0] == 0
        assert torch.equal(dE[none], start[none])


# ids of 9 bits a pass: one pass, two and three, on either side of the powers of two
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("vocab", [1, 300, 511, 512, 262143, 262144, 300007])
def test_embed_grad_of_sorted_tokens(ctx, vocab, accumulate):
    ids = torch.randint(0, vocab, (12001,), generator=gen(vocab), device=DEV)
    ids[torch.rand(len(ids), generator=gen(1), device=DEV) < 0.1] = -1
    _embed_grad(ctx, ids, vocab, 8, "bf16", accumulate)


@pytest.mark.parametrize("vocab", [(1 << 24) - 1, 1 << 24])
def test_embed_grad_of_a_short_list_over_a_wide_vocabulary(ctx, vocab):
    """Ids up to 2^24 - 2 are counted as floats; a wider vocabulary's are sorted."""
    ids = torch.randint(vocab - 40, vocab, (100,), generator=gen(1), device=DEV)
    ids[:3] = torch.tensor([0, vocab - 1, vocab - 2], device=DEV)
    _embed_grad(ctx, ids.int(), vocab, 1, "fp32", False)


@pytest.mark.parametrize("n", [10241, 300])
def test_embed_grad_reports_ids_outside_the_table(ctx, n):
    ids = torch.randint(0, 1000, (n,), generator=gen(1), device=DEV)
    ids[n // 2], ids[n - 1] = 1000, 1 << 40
    _embed_grad(ctx, ids, 1000, 8, "fp32", False, status=-1)


# ---- in a graph ----
@pytest.mark.parametrize("dt,T", [("bf16", 700), ("fp16", 40), ("fp32", 90)])
def test_the_ends_in_a_captured_graph(dt, T):
    """After a first call of the same sizes: a replay reads its inputs anew and gives a plain call's bits."""
    d, vocab = 136, 3001
    E, g, b = rnd(1, vocab, d, std=0.1, dt=dt), 1 + 0.1 * rnd(2, d), rnd(3, d)
    ids = torch.randint(-1, vocab, (T,), generator=gen(4), device=DEV)
    t = torch.randint(-1, vocab, (T,), generator=gen(5), device=DEV)
    x, y, dy, dx = (nans(T, d, dt=dt) for _ in range(4))
    m, s, dW, dg, db, mean = nans(T), nans(T), nans(vocab, d), nans(d), nans(d), torch.zeros(1, dtype=torch.float64, device=DEV)
    pair = torch.zeros(4, dtype=torch.float64, device=DEV)
    out = (y, dx, dW, dg, db, mean, pair)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        c = zo.Context(0)

        def run():
            zo.zoact_embed(c, E, ids, x, scale=8.0)
            zo.zoact_layer_norm(c, x, g, b, y, mean=m, rstd=s)
            zo.zoact_ce_pair(c, y[:T // 2 * 2], E, t[:T // 2], 0.5, pair)
            zo.zoact_ce_grad(c, y, E, t, dH=dy, dW=dW, mean=mean)
            zo.zoact_layer_norm_grad(c, dy, x, g, m, s, dX=dx, dgain=dg, dbias=db)
            zo.zoact_embed_grad(c, dx, ids, dW, scale=8.0, accumulate=True)

        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for step in range(3):
            ids.copy_(torch.randint(-1, vocab, (T,), generator=gen(10 + step), device=DEV))
            t.copy_(torch.randint(-1, vocab, (T,), generator=gen(20 + step), device=DEV))
            E.mul_(1.25)
            for o in out:
                o.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = [o.clone() for o in out]
            run()
            torch.cuda.synchronize()
            assert c.device_status() == 0
            assert all(torch.equal(a, o) for a, o in zip(got, out)) and float(mean) > 0
        c.close()
