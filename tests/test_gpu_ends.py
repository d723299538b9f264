"""The two ends of a language model on the GPU (C ABI) against the fp64 oracle: embedding rows and their gradient, layer
norm and its gradient, cross entropy of a head over the vocabulary with its gradient and the ZO estimates made of it.

Tolerances are bounds on the arithmetic: u is the unit roundoff of a stored type (bf16 2^-8, fp16 2^-11, fp32 2^-24), a sum
of k terms in fp32 errs by at most k 2^-24 times the sum of their magnitudes, and every result is rounded once to the
type that it is stored in (fp16 results below its normal range: by 2^-25).
"""
import numpy as np
import pytest
import torch

import paper_2607_01125_gb300 as zo
from oracle import ends

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
    g = torch.Generator(DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(TYPES[dt])


def ints(values, dtype=torch.int64):
    return torch.tensor(np.asarray(values), dtype=dtype, device=DEV)


def clean(ctx):
    torch.cuda.synchronize()
    assert ctx.device_status() == 0


def within(got, want, tol):
    err = np.abs(n64(got) - want)
    assert np.isfinite(n64(got)).all()
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


# ---- embedding ----
@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,d,vocab", [(1, 1, 1), (5, 7, 3), (100, 64, 1000), (33, 257, 50), (64, 4096, 300), (9, 5120, 20)])
def test_embed(ctx, dt, idt, n, d, vocab):
    rng = np.random.default_rng(n + d)
    ids = rng.integers(0, vocab, n)
    ids[rng.random(n) < 0.2] = -100
    E = rnd(1, vocab, d, dt=dt)
    Y = torch.full((n, d), float("nan"), dtype=TYPES[dt], device=DEV)
    zo.zoact_embed(ctx, E, ints(ids, idt), Y, scale=1.7)
    clean(ctx)
    want = (E.float()[torch.from_numpy(np.maximum(ids, 0)).to(DEV)] * 1.7) * ints(ids >= 0, torch.float32)[:, None]
    assert torch.equal(Y, want.to(TYPES[dt]))          # one product and one rounding: the same bits


def _embed_grad_case(ctx, dt, et, ids, d, vocab, accumulate, idt=torch.int64, scale=0.7):
    n = len(ids)
    dY = rnd(2, n, d, dt=dt)
    start = rnd(3, vocab, d, dt=et)
    dE = start.clone() if accumulate else torch.full((vocab, d), float("nan"), dtype=TYPES[et], device=DEV)
    zo.zoact_embed_grad(ctx, dY, ints(ids, idt), dE, scale=scale, accumulate=accumulate)
    clean(ctx)
    first = n64(start) if accumulate else None
    scale = float(np.float32(scale))
    want = ends.embed_grad(n64(dY), ids, vocab, scale, first)
    size = ends.embed_grad(np.abs(n64(dY)), ids, vocab, scale, None if first is None else np.abs(first))
    count = np.bincount([v for v in ids if v >= 0], minlength=vocab)[:, None]
    within(dE, want, (count + 3) * F * size + UNIT[et] * np.abs(want) * 1.01 + TINY[et])
    if accumulate:                                      # rows without a token are not touched
        none = torch.from_numpy(count[:, 0] == 0).to(DEV)
        assert torch.equal(dE[none], start[none])
    again = start.clone() if accumulate else torch.empty_like(dE)
    zo.zoact_embed_grad(ctx, dY, ints(ids, idt), again, scale=scale, accumulate=accumulate)
    clean(ctx)
    assert torch.equal(dE, again)


@pytest.mark.parametrize("dt,et", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,d,vocab", [(1, 1, 1), (3, 5, 2), (200, 40, 31), (1000, 72, 3000), (77, 1001, 200)])
def test_embed_grad(ctx, dt, et, accumulate, n, d, vocab):
    rng = np.random.default_rng(n + vocab)
    ids = rng.integers(0, vocab, n)
    ids[rng.random(n) < 0.1] = -1
    _embed_grad_case(ctx, dt, et, list(ids), d, vocab, accumulate)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind", ["one id", "two ids", "none", "last row", "runs", "int32 wide"])
def test_embed_grad_of_uneven_ids(ctx, kind, accumulate):
    rng = np.random.default_rng(5)
    n, vocab, idt = 3000, 70001, torch.int64
    if kind == "one id":
        ids = np.full(n, 12345)
    elif kind == "two ids":
        ids = np.where(rng.random(n) < 0.5, 65535, 65536)
    elif kind == "none":
        ids = np.full(n, -100)
    elif kind == "last row":
        ids = np.full(n, vocab - 1)
        ids[0] = 0
    elif kind == "runs":                                # lengths around every multiple of 16 up to 130
        ids = np.repeat(np.arange(48) * 1459, [1 + (i * 16 + j) % 130 for i in range(16) for j in (15, 16, 17)])
        rng.shuffle(ids)
    else:
        ids, idt = rng.integers(0, vocab, 20011), torch.int32
    _embed_grad_case(ctx, "bf16", "bf16", list(ids), 24, vocab, accumulate, idt)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n", [10239, 10240, 10241, 40000])
def test_embed_grad_of_long_lists(ctx, n, accumulate):
    """Both ways to order the tokens, with ids as frequent as 1 / rank (the first has a tenth of them) and unfrequent ones."""
    rng = np.random.default_rng(n)
    vocab = 50003
    ids = np.exp(rng.random(n) * np.log(vocab)).astype(np.int64) * 7919 % vocab
    ids[rng.random(n) < 0.1] = -1
    _embed_grad_case(ctx, "fp16", "fp32", list(ids), 8, vocab, accumulate)


def test_embed_of_no_tokens(ctx):
    E, none = rnd(1, 5, 8), ints([], torch.int64)
    zo.zoact_embed(ctx, E, none, torch.empty(0, 8, device=DEV))
    dE = torch.ones(5, 8, device=DEV)
    zo.zoact_embed_grad(ctx, torch.empty(0, 8, device=DEV), none, dE, accumulate=True)
    clean(ctx)
    assert (dE == 1).all()
    zo.zoact_embed_grad(ctx, torch.empty(0, 8, device=DEV), none, dE)
    clean(ctx)
    assert (dE == 0).all()


def test_ids_outside_the_table_are_no_tokens_and_are_reported(ctx):
    E, ids = rnd(1, 10, 8), ints([3, 10, 2 ** 40, -5])
    Y = torch.full((4, 8), float("nan"), device=DEV)
    zo.zoact_embed(ctx, E, ids, Y)
    torch.cuda.synchronize()
    assert ctx.device_status() == -1 and torch.equal(Y[0], E[3]) and (Y[1:] == 0).all()
    dE = torch.full((10, 8), float("nan"), device=DEV)
    zo.zoact_embed_grad(ctx, torch.ones(4, 8, device=DEV), ids, dE)
    torch.cuda.synchronize()
    assert ctx.device_status() == -1
    assert (dE[3] == 1).all() and dE.sum() == 8
    loss = torch.empty(4, device=DEV)
    zo.zoact_ce_loss(ctx, rnd(2, 4, 8), E, ids, loss=loss)
    torch.cuda.synchronize()
    assert ctx.device_status() == -1 and loss[0] > 0 and (loss[1:] == 0).all()


# ---- layer norm ----
NORM_SIZES = [(1, 1), (3, 2), (5, 33), (64, 64), (7, 1000), (300, 1001), (40, 4096), (9, 5120), (4, 8200), (3, 20480), (2, 40001)]


def _depth(n):
    return n / 32 + 16                                   # terms in a row on one thread, and the joins


def _norm_and_grad(ctx, X, dY, g, b, dt, eps=1e-5):
    """Layer norm of X and its gradient, each output within its bound; returns the gradient's outputs and a call that
    asks for some of them."""
    rows, n = X.shape
    Y = torch.full((rows, n), float("nan"), dtype=X.dtype, device=DEV)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    zo.zoact_layer_norm(ctx, X, g, b, Y, eps=eps, mean=mean, rstd=rstd)
    clean(ctx)
    x, gg, bb = n64(X), n64(g), n64(b)
    wy, wm, ws = ends.layer_norm(x, gg, bb, float(np.float32(eps)))
    k = _depth(n)
    em = k * F * np.abs(x).mean(axis=1) + F * np.abs(wm)
    within(mean, wm, em)
    es = (2 * k + 8) * F + (ws * em) ** 2                # relative, of rstd
    within(rstd, ws, es * ws)
    xh = np.abs(x - wm[:, None]) * ws[:, None]
    ty = np.abs(gg) * (ws[:, None] * em[:, None] + xh * (es[:, None] + 3 * F)) + 2 * F * (np.abs(wy) + np.abs(bb))
    within(Y, wy, ty + UNIT[dt] * (np.abs(wy) + ty) + TINY[dt])

    dX = torch.full((rows, n), float("nan"), dtype=X.dtype, device=DEV)
    dg, db = torch.full((n,), float("nan"), device=DEV), torch.full((n,), float("nan"), device=DEV)

    def grad(**outputs):
        zo.zoact_layer_norm_grad(ctx, dY, X, g, mean, rstd, **outputs)
        clean(ctx)

    grad(dX=dX, dgain=dg, dbias=db)
    dy, m, s = n64(dY), n64(mean), n64(rstd)
    wx, wg, wb = ends.layer_norm_grad(dy, x, gg, m, s)
    xh, u = (x - m[:, None]) * s[:, None], dy * gg
    c1, c2 = np.abs(u).mean(axis=1, keepdims=True), np.abs(u * xh).mean(axis=1, keepdims=True)
    tx = s[:, None] * ((k + 8) * F * (c1 + np.abs(xh) * c2) + 8 * F * np.abs(u))
    within(dX, wx, tx + UNIT[dt] * (np.abs(wx) + tx) + TINY[dt])
    within(dg, wg, (rows + 8) * F * np.abs(dy * xh).sum(axis=0))
    within(db, wb, (rows + 8) * F * np.abs(dy).sum(axis=0))
    return dX, dg, db, grad


@pytest.mark.parametrize("dt,pt", [("fp32", "fp32"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp16", "fp16"), ("fp16", "fp32")])
@pytest.mark.parametrize("rows,n", NORM_SIZES)
def test_layer_norm_and_its_gradient(ctx, dt, pt, rows, n):
    X = (rnd(1, rows, n) * torch.exp(rnd(2, rows, 1)) + 3 * rnd(3, rows, 1)).to(TYPES[dt])
    g, b = (1 + 0.3 * rnd(4, n)).to(TYPES[pt]), rnd(5, n, dt=pt)
    dX, dg, db, grad = _norm_and_grad(ctx, X, rnd(6, rows, n, dt=dt), g, b, dt)
    # each output alone, the others not asked for: the same bits
    dX1, dg1, db1 = torch.empty_like(dX), torch.empty_like(dg), torch.empty_like(db)
    grad(dX=dX1), grad(dgain=dg1), grad(dbias=db1)
    assert torch.equal(dX, dX1) and torch.equal(dg, dg1) and torch.equal(db, db1)


def test_layer_norm_gradient_of_many_rows(ctx):
    rows, n = 5003, 264
    X, dY = rnd(1, rows, n, dt="bf16"), rnd(2, rows, n, dt="bf16")
    mean, rstd = 0.01 * rnd(3, rows), 1 + 0.01 * rnd(4, rows)
    dX, dg, db = torch.empty_like(X), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    zo.zoact_layer_norm_grad(ctx, dY, X, None, mean, rstd, dX=dX, dgain=dg, dbias=db)
    clean(ctx)
    x, dy, m, s = n64(X), n64(dY), n64(mean), n64(rstd)
    wx, wg, wb = ends.layer_norm_grad(dy, x, None, m, s)
    xh = (x - m[:, None]) * s[:, None]
    within(dg, wg, (rows + 8) * F * np.abs(dy * xh).sum(axis=0))
    within(db, wb, (rows + 8) * F * np.abs(dy).sum(axis=0))
    c = np.abs(dy).mean(axis=1, keepdims=True) + np.abs(xh) * np.abs(dy * xh).mean(axis=1, keepdims=True)
    tx = s[:, None] * ((_depth(n) + 8) * F * c + 8 * F * np.abs(dy))
    within(dX, wx, tx + UNIT["bf16"] * (np.abs(wx) + tx))


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("n,ld,off", [(64, 72, 8), (1001, 1003, 1), (4096, 4100, 3)])
def test_layer_norm_of_strided_rows(ctx, dt, n, ld, off):
    wide, wdy = rnd(1, 50, ld + off, dt=dt), rnd(2, 50, ld + off, dt=dt)
    _norm_and_grad(ctx, wide[:, off:off + n], wdy[:, off:off + n], 1 + 0.3 * rnd(3, n), rnd(4, n), dt)


def test_layer_norm_of_constant_rows_and_of_no_rows(ctx):
    X = torch.full((3, 96), 7.25, device=DEV)
    Y, rstd = torch.empty_like(X), torch.empty(3, device=DEV)
    b = rnd(1, 96)
    zo.zoact_layer_norm(ctx, X, None, b, Y, eps=1e-4, rstd=rstd)
    clean(ctx)
    assert torch.equal(Y, b.expand(3, 96)) and torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-6, atol=0)
    none = torch.empty(0, 96, device=DEV)
    stat = torch.empty(0, device=DEV)
    zo.zoact_layer_norm(ctx, none, None, b, torch.empty_like(none), mean=stat, rstd=stat)
    dg, db = torch.ones(96, device=DEV), torch.ones(96, device=DEV)
    zo.zoact_layer_norm_grad(ctx, none, none, None, stat, stat, dX=torch.empty_like(none), dgain=dg, dbias=db)
    clean(ctx)
    assert (dg == 0).all() and (db == 0).all()


# ---- cross entropy ----
def _targets(rng, T, vocab, ignored):
    t = rng.integers(0, vocab, T)
    t[rng.random(T) < ignored] = -100
    return t


def _logit_error(h, w):
    """A bound on a logit's error: d products summed in fp32."""
    return (h.shape[1] + 8) * F * (np.abs(h) @ np.abs(w).T).max()


CE_SIZES = [(1, 8, 1), (1, 8, 300), (3, 64, 7), (16, 256, 1009), (33, 512, 2000), (130, 128, 513), (257, 264, 1777),
            (300, 1024, 640), (64, 4096, 256), (520, 72, 3001)]


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T,d,vocab", CE_SIZES)
def test_cross_entropy_and_its_gradient(ctx, dt, T, d, vocab):
    rng = np.random.default_rng(T + d)
    H, W = rnd(1, T, d, dt=dt), rnd(2, vocab, d, std=2.0 / np.sqrt(d), dt=dt)
    t = _targets(rng, T, vocab, 0.2)
    loss, lse, mean = (torch.full((T,), float("nan"), device=DEV), torch.full((T,), float("nan"), device=DEV),
                       torch.full((1,), float("nan"), dtype=torch.float64, device=DEV))
    zo.zoact_ce_loss(ctx, H, W, ints(t), loss=loss, lse=lse, mean=mean)
    clean(ctx)
    h, w = n64(H), n64(W)
    wloss, wlse, wmean = ends.cross_entropy(h, w, t)
    ez = _logit_error(h, w)
    el = 2 * ez + 2.0 ** -20 + 4 * F * np.abs(wlse)     # both logits' errors, the exponentials' and the sum's, the rounding
    within(lse, wlse, el)
    within(loss, wloss, el + F * np.abs(wloss))
    assert (n64(loss)[t < 0] == 0).all()
    within(mean, wmean, el.max())

    for wt in {dt, "fp32"}:
        dH, dW = torch.full_like(H, float("nan")), torch.full((vocab, d), float("nan"), dtype=TYPES[wt], device=DEV)
        loss2, lse2, mean2 = torch.empty_like(loss), torch.empty_like(lse), torch.empty_like(mean)
        zo.zoact_ce_grad(ctx, H, W, ints(t), dH=dH, dW=dW, loss=loss2, lse=lse2, mean=mean2, grad_scale=3.0)
        clean(ctx)
        assert torch.equal(loss, loss2) and torch.equal(lse, lse2) and torch.equal(mean, mean2)
        wh, ww = ends.cross_entropy_grad(h, w, t, 3.0)
        N = max(1, int((t >= 0).sum()))
        z = h @ w.T
        P = np.exp(z - wlse[:, None]) * (t >= 0)[:, None]
        G = P.copy()
        G[np.arange(T), np.maximum(t, 0)] -= (t >= 0)
        # an element of G errs by its rounding to the operand's type (once, and once on its way in fp16; fp32: three
        # parts of it), by the logit's and lse's errors, and where it is tiny beside its tile's largest by 2^-25 of that
        ug = 2.0 ** -21 if dt == "fp32" else 1.01 * UNIT[dt] + 2.0 ** -11
        eg = ug * np.abs(G) + (2 * ez + 2.0 ** -20) * P + (0 if dt == "fp32" else 2.0 ** -25) * (t >= 0)[:, None]
        th = 3.0 / N * (eg @ np.abs(w) + (vocab + 8) * F * (np.abs(G) @ np.abs(w)))
        tw = 3.0 / N * (eg.T @ np.abs(h) + (T + 8) * F * (np.abs(G).T @ np.abs(h)))
        within(dH, wh, th + UNIT[dt] * (np.abs(wh) + th) + TINY[dt])
        within(dW, ww, tw + UNIT[wt] * (np.abs(ww) + tw) + TINY[wt])
        assert (n64(dH)[t < 0] == 0).all()
        if wt == "fp32":
            twice = dW.clone()
            zo.zoact_ce_grad(ctx, H, W, ints(t), dW=twice, grad_scale=3.0, accumulate=True)
            clean(ctx)
            within(twice, 2 * ww, 2 * tw + 4 * F * np.abs(ww))
        alone = torch.full_like(dH, float("nan"))
        zo.zoact_ce_grad(ctx, H, W, ints(t, torch.int32), dH=alone, grad_scale=3.0)
        clean(ctx)
        assert torch.equal(alone, dH)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("nb", [1, 2, 3, 9])
def test_cross_entropy_of_evaluation_blocks(ctx, dt, nb):
    T, d, vocab = 70, 128, 600
    rng = np.random.default_rng(nb)
    H0 = rnd(1, T, d)
    H = torch.cat([H0 + 0.05 * rnd(10 + b, T, d) for b in range(nb)]).to(TYPES[dt])
    W, t = rnd(2, vocab, d, std=0.2, dt=dt), _targets(rng, T, vocab, 0.3)
    loss, mean = torch.empty(nb * T, device=DEV), torch.empty(nb, dtype=torch.float64, device=DEV)
    zo.zoact_ce_loss(ctx, H, W, ints(t), n_blocks=nb, loss=loss, mean=mean)
    h, w = n64(H), n64(W)
    wloss, wlse, wmean = ends.cross_entropy(h, w, t, nb)
    el = 2 * _logit_error(h, w) + 2.0 ** -20 + 4 * F * np.abs(wlse).max()
    within(loss, wloss, el)
    within(mean, wmean, el)
    if nb == 2:
        out = torch.empty(4, dtype=torch.float64, device=DEV)
        zo.zoact_ce_pair(ctx, H, W, ints(t), 1e-3, out)
        clean(ctx)
        within(out, ends.pair(wmean, wloss, t, float(np.float32(1e-3))), np.array([el, el, 2 * el, 2 * el / 2e-3 * 1.001]))
        o, m = n64(out), n64(mean)
        assert o[0] == m[0] and o[1] == m[1]
        rows = n64(loss)
        D = (rows[:T] - rows[T:]).sum() / max(1, (t >= 0).sum())
        assert abs(o[2] - D) <= 1e-13 * np.abs(rows).max() and abs(o[3] - D / (2 * float(np.float32(1e-3)))) <= 1e-9
    if nb > 1:
        out = torch.empty(2 * nb - 1, dtype=torch.float64, device=DEV)
        zo.zoact_ce_multi(ctx, H, W, ints(t), nb, 0.5, out)
        clean(ctx)
        within(out, np.concatenate([wmean, (wmean[1:] - wmean[0]) / 0.5]), np.repeat([el, 4 * el], [nb, nb - 1]))
    clean(ctx)


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
def test_cross_entropy_of_large_and_of_equal_logits(ctx, dt):
    # rows with one logit far above the others (+ or - 4000), rows of equal logits, a row whose target is far below the rest
    d, vocab = 16, 700
    H, W = torch.zeros(5, d, device=DEV), torch.zeros(vocab, d, device=DEV)
    W[3, 0] = W[650, 1] = 64.0
    H[0, 0], H[1, 0], H[2, 1], H[4, 1] = 62.5, -62.5, 62.5, 62.5
    t = ints([3, 3, 650, 5, 0])
    H, W = H.to(TYPES[dt]), W.to(TYPES[dt])
    loss, lse = torch.empty(5, device=DEV), torch.empty(5, device=DEV)
    dH, dW = torch.empty_like(H), torch.empty_like(W)
    zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=dW, loss=loss, lse=lse)
    clean(ctx)
    rest = np.log(vocab - 1)
    within(loss, np.array([0, 4000 + rest, 0, np.log(vocab), 4000]), np.array([1e-3, 2e-3, 1e-3, 1e-5, 1e-3]))
    wh, ww = ends.cross_entropy_grad(n64(H), n64(W), n64(t).astype(int))
    within(dH, wh, 2.0 ** -6 * np.abs(wh) + 1e-4)
    within(dW, ww, 2.0 ** -6 * np.abs(ww) + 1e-4)


def test_cross_entropy_without_a_counted_row(ctx):
    H, W, t = rnd(1, 6, 32, dt="bf16"), rnd(2, 90, 32, dt="bf16"), ints([-100] * 6)
    loss, mean = torch.ones(6, device=DEV), torch.ones(1, dtype=torch.float64, device=DEV)
    dH, dW = torch.ones_like(H), torch.ones_like(W)
    zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=dW, loss=loss, mean=mean)
    clean(ctx)
    assert (loss == 0).all() and mean[0] == 0 and (dH == 0).all() and (dW == 0).all()
    none = ints([], torch.int64)
    mean.fill_(1), dW.fill_(1)
    zo.zoact_ce_grad(ctx, H[:0], W, none, dH=dH[:0], dW=dW, mean=mean)
    clean(ctx)
    assert mean[0] == 0 and (dW == 0).all()
    out = torch.ones(4, dtype=torch.float64, device=DEV)
    zo.zoact_ce_pair(ctx, H[:0], W, none, 1e-3, out)
    clean(ctx)
    assert (out == 0).all()


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T", [40, 700])
def test_cross_entropy_of_ignored_rows_that_are_not_finite(ctx, dt, T):
    """What lies in a row without a target reaches no output: the same bits as with zeros there."""
    d, vocab = 128, 700
    rng = np.random.default_rng(T)
    t = _targets(rng, T, vocab, 0.3)
    t[[0, T - 1]] = -1
    H, W = rnd(1, T, d, dt=dt), rnd(2, vocab, d, std=0.2, dt=dt)
    out = []
    for fill in (0.0, float("nan"), float("inf"), torch.finfo(TYPES[dt]).min):
        h = H.clone()
        h[torch.as_tensor(t < 0, device=DEV)] = fill
        dH, dW = torch.empty_like(h), torch.empty_like(W)
        loss, mean = torch.empty(T, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
        zo.zoact_ce_grad(ctx, h, W, ints(t), dH=dH, dW=dW, loss=loss, mean=mean)
        clean(ctx)
        out.append((dH, dW, loss, mean))
    assert all(torch.isfinite(x).all() for x in out[0])
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))


@pytest.mark.parametrize("T,d,vocab", [(2, 1024, 20000), (24, 260, 20011), (25, 260, 20011), (160, 64, 900), (9, 5124, 130)])
def test_cross_entropy_of_fp32_rows_multiplied_as_they_are_or_in_parts(ctx, T, d, vocab):
    """Both sides of the rule by rows and by blocks, and a width whose rows do not fit; the gradient call gives the same bits."""
    rng = np.random.default_rng(T + vocab)
    H, W = rnd(1, T, d), rnd(2, vocab, d, std=2.0 / np.sqrt(d))
    t = _targets(rng, T, vocab, 0.1)
    loss, lse, mean = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
    zo.zoact_ce_loss(ctx, H, W, ints(t), loss=loss, lse=lse, mean=mean)
    loss2, dH = torch.empty_like(loss), torch.empty_like(H)
    zo.zoact_ce_grad(ctx, H, W, ints(t), dH=dH, loss=loss2)
    clean(ctx)
    h, w = n64(H), n64(W)
    wloss, wlse, wmean = ends.cross_entropy(h, w, t)
    ez = _logit_error(h, w)
    el = 2 * ez + 2.0 ** -20 + 4 * F * np.abs(wlse)
    within(lse, wlse, el)
    within(loss, wloss, el + F * np.abs(wloss))
    within(mean, wmean, el.max())
    assert torch.equal(loss, loss2)
    P = np.exp(h @ w.T - wlse[:, None]) * (t >= 0)[:, None]
    G = P.copy()
    G[np.arange(T), np.maximum(t, 0)] -= (t >= 0)
    eg = 2.0 ** -21 * np.abs(G) + (2 * ez + 2.0 ** -20) * P
    wh, N = ends.cross_entropy_grad(h, w, t)[0], max(1, int((t >= 0).sum()))
    within(dH, wh, (eg @ np.abs(w) + (vocab + 8) * F * (np.abs(G) @ np.abs(w))) / N + F * np.abs(wh))


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
def test_cross_entropy_gradient_beside_a_target_that_is_nearly_sure(ctx, dt):
    """Logits 24 below the target's, in its tile of the vocabulary too: their rows of dW keep their own digits, and the loss
    those that a sum beside 1 can have."""
    T, d, vocab = 6, 256, 700
    W = rnd(1, vocab, d, std=1.0 / 16, dt=dt)
    t = np.array([0, 1, 130, 400, 640, 699])
    w = n64(W)
    H = torch.as_tensor(24.0 * w[t] / (w[t] ** 2).sum(axis=1, keepdims=True), device=DEV).to(TYPES[dt])
    dW, loss = torch.empty(vocab, d, device=DEV), torch.empty(T, device=DEV)
    zo.zoact_ce_grad(ctx, H, W, ints(t), dW=dW, loss=loss)
    clean(ctx)
    h = n64(H)
    z = h @ w.T
    wloss, wlse, _ = ends.cross_entropy(h, w, t)
    ez = _logit_error(h, w)
    P = np.exp(z - wlse[:, None])
    P[np.arange(T), t] = 0
    S = P.sum(axis=1)                                   # 1 - the target's share, to S^2
    assert S.max() < 1e-6
    within(loss, S, 130 * F + (2 * ez + 2.0 ** -20) * S)    # a tile's 128 exponentials summed beside a 1
    others = np.setdiff1d(np.arange(vocab), t)
    want = (P.T @ h / T)[others]
    ug = 2.0 ** -21 if dt == "fp32" else 1.01 * UNIT[dt] + 2.0 ** -11
    # fp16's G lies on multiples of 2^-24 of its scale 2^15
    eg = (ug + 2 * ez + 2.0 ** -20) * P + (2.0 ** -40 if dt == "fp16" else 0)
    within(dW[torch.as_tensor(others, device=DEV)], want, ((eg.T @ np.abs(h) + (T + 8) * F * (P.T @ np.abs(h))) / T)[others])


def test_cross_entropy_of_non_finite_rows(ctx):
    H, W, t = rnd(1, 40, 64, dt="bf16"), rnd(2, 500, 64, dt="bf16"), ints(np.arange(40))
    H[7, 3] = float("nan")
    loss, mean = torch.empty(40, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
    zo.zoact_ce_loss(ctx, H, W, t, loss=loss, mean=mean)
    torch.cuda.synchronize()
    assert ctx.device_status() == -4
    assert torch.isnan(loss[7]) and torch.isfinite(loss[torch.arange(40, device=DEV) != 7]).all() and torch.isnan(mean[0])


@pytest.mark.parametrize("dt,wt", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
def test_cross_entropy_gradient_in_several_chunks_of_rows(ctx, dt, wt):
    # a vocabulary so wide that the gradient by the logits of 2 GiB holds fewer rows than there are
    vocab, d = 1 << 20, 8
    T = 1100 if dt == "bf16" else 300
    rng = np.random.default_rng(4)
    t = torch.from_numpy(_targets(rng, T, vocab, 0.1)).to(DEV)
    H, W = rnd(1, T, d, dt=dt), rnd(2, vocab, d, std=0.5, dt=dt)
    dH, dW = torch.empty_like(H), torch.empty(vocab, d, dtype=TYPES[wt], device=DEV)
    loss = torch.empty(T, device=DEV)
    zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=dW, loss=loss)
    clean(ctx)
    h, w = H.double(), W.double()
    wh, ww, N = torch.empty_like(h), torch.zeros_like(w), int((t >= 0).sum())
    size_h, size_w = torch.empty_like(h), torch.zeros_like(w)
    for r in range(0, T, 100):
        z = h[r:r + 100] @ w.t()
        lp = torch.log_softmax(z, dim=1)
        tr = t[r:r + 100]
        at = torch.arange(len(tr), device=DEV)
        want = torch.where(tr >= 0, -lp[at, tr.clamp(min=0)], torch.zeros(len(tr), dtype=torch.float64, device=DEV))
        assert (loss[r:r + 100].double() - want).abs().max() < 1e-4
        G = lp.exp()
        G[at, tr.clamp(min=0)] -= 1
        G *= (tr >= 0)[:, None] / N
        wh[r:r + 100], size_h[r:r + 100] = G @ w, G.abs() @ w.abs()
        ww += G.t() @ h[r:r + 100]
        size_w += G.abs().t() @ h[r:r + 100].abs()
    # 2^20 (or T) terms: their roundings to the operand's type are independent, and 2^-12 of the magnitudes covers the sums
    rel = 2.0 ** -14 if dt == "fp32" else 1.2 * UNIT[dt] + 2.0 ** -12
    assert ((dH.double() - wh).abs() <= (rel + UNIT[dt]) * size_h + 1e-9).all()
    assert ((dW.double() - ww).abs() <= (rel + UNIT[wt]) * size_w + 1e-12).all()


def test_cross_entropy_gradient_against_differences_of_the_loss(ctx):
    T, d, vocab = 48, 64, 333
    H, W = rnd(1, T, d), rnd(2, vocab, d, std=0.3)
    t = ints(_targets(np.random.default_rng(1), T, vocab, 0.2))
    dH, dW = torch.empty_like(H), torch.empty_like(W)
    zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=dW)
    A, B = rnd(3, T, d), rnd(4, vocab, d)
    mean = torch.empty(1, dtype=torch.float64, device=DEV)

    def L(step):
        zo.zoact_ce_loss(ctx, H + step * A, W + step * B, t, mean=mean)
        return float(mean)

    # central differences: an error of step^2 times the third derivative (logits move by about step * (0.3 * 8 + 8 + ...)),
    # and the losses' own 1e-6 / step
    step = 2.0 ** -9
    slope = (L(step) - L(-step)) / (2 * step)
    want = float((dH.double() * A.double()).sum() + (dW.double() * B.double()).sum())
    clean(ctx)
    assert abs(slope - want) < 5e-3 * max(1.0, abs(want))


# ---- use ----
def test_the_ends_run_on_a_stream_of_their_own(ctx):
    T, d, vocab = 40, 64, 500
    E, g, b = rnd(1, vocab, d, dt="bf16"), 1 + 0.1 * rnd(2, d), rnd(3, d)
    ids, t = ints(np.arange(T) * 7 % vocab), ints(np.arange(T) * 11 % vocab)

    def run():
        x, y = torch.empty(T, d, dtype=torch.bfloat16, device=DEV), torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
        m, s, dy, dx = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty_like(x), torch.empty_like(x)
        dW, dg, db, mean = torch.empty_like(E), torch.empty_like(g), torch.empty_like(b), torch.empty(1, dtype=torch.float64, device=DEV)
        zo.zoact_embed(ctx, E, ids, x, scale=8.0)
        zo.zoact_layer_norm(ctx, x, g, b, y, mean=m, rstd=s)
        zo.zoact_ce_grad(ctx, y, E, t, dH=dy, dW=dW, mean=mean)
        zo.zoact_layer_norm_grad(ctx, dy, x, g, m, s, dX=dx, dgain=dg, dbias=db)
        dE = dW.float()
        zo.zoact_embed_grad(ctx, dx, ids, dE, scale=8.0, accumulate=True)
        return [mean, dE, dg, db]

    want = run()
    clean(ctx)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.sync_stream()
        got = run()
    torch.cuda.synchronize()
    ctx.sync_stream()
    assert all(torch.equal(a, c) for a, c in zip(want, got))


def test_refusals(ctx):
    f, h = rnd(1, 8, 16), rnd(2, 8, 16, dt="bf16")
    W, t = rnd(3, 20, 16), ints(np.arange(8))
    loss, mean = torch.empty(8, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
    before = ctx.launch_count()

    def refused(fn, status=None):
        with pytest.raises(zo.ZoactError if status is not None else (ValueError, KeyError)) as e:
            fn()
        if status is not None:
            assert e.value.status == status

    refused(lambda: zo.zoact_ce_loss(ctx, f, W, t), -1)                                      # no output
    refused(lambda: zo.zoact_ce_grad(ctx, f, W, t), -1)
    refused(lambda: zo.zoact_ce_loss(ctx, f[:, :6].contiguous(), W[:, :6].contiguous(), t, loss=loss), -1)   # d % 4
    refused(lambda: zo.zoact_ce_loss(ctx, h[:, :12].contiguous(), W[:, :12].to(torch.bfloat16), t, loss=loss), -1)   # d % 8
    refused(lambda: zo.zoact_ce_grad(ctx, h, W.to(torch.bfloat16), t, dW=W.to(torch.bfloat16), accumulate=True), -2)
    refused(lambda: zo.zoact_ce_pair(ctx, f, W, t[:4], 0.0, torch.empty(4, dtype=torch.float64, device=DEV)), -1)
    refused(lambda: zo.zoact_ce_multi(ctx, f, W, t, 1, 1.0, torch.empty(1, dtype=torch.float64, device=DEV)), -1)
    refused(lambda: zo.zoact_ce_loss(ctx, f, W, t[:7], loss=loss))                            # rows and targets
    refused(lambda: zo.zoact_ce_loss(ctx, f, W.to(torch.bfloat16), t, loss=loss))             # two types
    refused(lambda: zo.zoact_ce_loss(ctx, f, W, t.float(), loss=loss))                        # float targets
    refused(lambda: zo.zoact_ce_loss(ctx, f, W, t, mean=mean.float()))                        # fp32 mean
    refused(lambda: zo.zoact_ce_loss(ctx, f.t().contiguous().t(), W, t, loss=loss))           # column-major
    refused(lambda: zo.zoact_ce_loss(ctx, f.double(), W.double(), t, loss=loss))              # fp64
    refused(lambda: zo.zoact_ce_grad(ctx, f, W, t, dW=W.to(torch.bfloat16)), -1)              # 16-bit dW of fp32
    refused(lambda: zo.zoact_layer_norm(ctx, f, None, None, f.clone(), eps=-1.0), -1)
    refused(lambda: zo.zoact_layer_norm(ctx, f, rnd(1, 16, dt="bf16"), None, f.clone()), -1)   # 16-bit gain of fp32
    refused(lambda: zo.zoact_layer_norm(ctx, f, rnd(1, 16), rnd(1, 15), f.clone()))
    refused(lambda: zo.zoact_layer_norm(ctx, f, None, None, h))
    refused(lambda: zo.zoact_layer_norm(ctx, f.t(), None, None, torch.empty(16, 8, device=DEV)))
    refused(lambda: zo.zoact_layer_norm_grad(ctx, f, f, None, loss, loss), -1)                # no output
    refused(lambda: zo.zoact_layer_norm_grad(ctx, f[:4], f, None, loss, loss, dX=f.clone()))
    refused(lambda: zo.zoact_embed(ctx, f, t, f[:4].clone()))
    refused(lambda: zo.zoact_embed(ctx, f, t.float(), f.clone()))
    refused(lambda: zo.zoact_embed_grad(ctx, f, t, W.to(torch.bfloat16)), -1)                 # 16-bit dE of fp32 dY
    refused(lambda: zo.zoact_embed_grad(ctx, f[:4], t, W.clone()))
    assert ctx.launch_count() == before
    clean(ctx)
