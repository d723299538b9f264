"""Cross entropy where entries of the vocabulary are masked by their logits: minus infinity, and the type's lowest value.

A masked entry has a share of exp(-inf) = 0 in its row: the losses and gradients are those of the vocabulary without it, whole
tiles of masked entries included.  The mask is a constant feature of the hidden states (column 0), whose weight is 0 for
the entries that stay.  Tolerances: F = 2^-24; a logit is a sum of d products in fp32, a loss two logits and the sum of the
exponentials, G is rounded to the operands' type (bf16 2^-8, fp16 2^-11; fp32: three parts), a result to its own.
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


def ints(values):
    return torch.tensor(np.asarray(values), dtype=torch.int64, device=DEV)


def within(got, want, tol):
    got = n64(got)
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    assert (err <= tol).all(), float((err / np.maximum(tol, 1e-300)).max())


def _masked(dt, T, d, vocab, feature, weight):
    """H, W, targets and which entries stay: a third of them and every entry of the second to fourth 128 and of the last ones
    masked."""
    rng = np.random.default_rng(T + vocab)
    H, W = rnd(1, T, d, dt=dt), rnd(2, vocab, d, std=2.0 / np.sqrt(d), dt=dt)
    stay = rng.random(vocab) > 1 / 3
    stay[128:512] = False
    stay[vocab - 150:] = False
    stay[[0, 600]] = True
    H[:, 0] = feature
    W[:, 0] = 0.0
    W[torch.as_tensor(~stay, device=DEV), 0] = weight
    t = rng.choice(np.flatnonzero(stay), T)
    t[rng.random(T) < 0.2] = -1
    return H, W, t, stay


def _against_the_rest(ctx, H, W, t, stay, dt, grad):
    """The losses (and gradients) against the oracle's on the entries that stay."""
    T, d = H.shape
    loss, lse, mean = (torch.full((T,), float("nan"), device=DEV), torch.full((T,), float("nan"), device=DEV),
                       torch.full((1,), float("nan"), dtype=torch.float64, device=DEV))
    zo.zoact_ce_loss(ctx, H, W, ints(t), loss=loss, lse=lse, mean=mean)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    at = np.cumsum(stay) - 1                             # an entry's place among those that stay
    tr = np.where(t >= 0, at[np.maximum(t, 0)], -1)
    h, w = n64(H), n64(W)[stay]
    wloss, wlse, wmean = ends.cross_entropy(h, w, tr)
    ez = (d + 8) * F * (np.abs(h) @ np.abs(w).T).max()
    el = 2 * ez + 2.0 ** -20 + 4 * F * np.abs(wlse)
    within(lse, wlse, el)
    within(loss, wloss, el + F * np.abs(wloss))
    within(mean, wmean, el.max())
    if not grad:
        return
    dH, dW = torch.full_like(H, float("nan")), torch.full_like(W, float("nan"))
    loss2, lse2 = torch.empty_like(loss), torch.empty_like(lse)
    zo.zoact_ce_grad(ctx, H, W, ints(t), dH=dH, dW=dW, loss=loss2, lse=lse2)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    wh, ww = ends.cross_entropy_grad(h, w, tr)
    N = max(1, int((t >= 0).sum()))
    P = np.exp(h @ w.T - wlse[:, None]) * (t >= 0)[:, None]
    G = P.copy()
    G[np.arange(T), np.maximum(tr, 0)] -= (t >= 0)
    ug = 2.0 ** -21 if dt == "fp32" else 1.01 * UNIT[dt] + 2.0 ** -11
    eg = ug * np.abs(G) + (2 * ez + 2.0 ** -20) * P + (0 if dt == "fp32" else 2.0 ** -25) * (t >= 0)[:, None]
    th = (eg @ np.abs(w) + (len(stay) + 8) * F * (np.abs(G) @ np.abs(w))) / N
    tw = (eg.T @ np.abs(h) + (T + 8) * F * (np.abs(G).T @ np.abs(h))) / N
    within(dH, wh, th + UNIT[dt] * (np.abs(wh) + th) + TINY[dt])
    keep = torch.as_tensor(stay, device=DEV)
    within(dW[keep], ww, tw + UNIT[dt] * (np.abs(ww) + tw) + TINY[dt])
    assert (dW[~keep] == 0).all()


# fp32: a few rows, multiplied as they are (the parts that more rows are multiplied in hold no infinity)
@pytest.mark.parametrize("dt,T,d,vocab", [("bf16", 3, 64, 700), ("fp16", 40, 136, 1500), ("bf16", 601, 520, 20011),
                                          ("fp32", 5, 64, 1500)])
def test_entries_masked_by_minus_infinity(ctx, dt, T, d, vocab):
    H, W, t, stay = _masked(dt, T, d, vocab, 1.0, -float("inf"))
    _against_the_rest(ctx, H, W, t, stay, dt, grad=False)


# the weights stay finite, so that 0 times them is 0 in dH; 2^129 overflows in the sum
@pytest.mark.parametrize("dt,T,d,vocab", [("bf16", 3, 64, 700), ("bf16", 40, 136, 1500), ("bf16", 601, 520, 20011),
                                          ("fp32", 5, 64, 1500), ("fp32", 90, 72, 5000)])
def test_entries_whose_logits_overflow_to_minus_infinity(ctx, dt, T, d, vocab):
    H, W, t, stay = _masked(dt, T, d, vocab, 4.0, -2.0 ** 127)
    _against_the_rest(ctx, H, W, t, stay, dt, grad=True)


# fp32 above bf16's largest value, 3.3895e38: what the first of three bf16 parts would round to infinity
@pytest.mark.parametrize("T,d,vocab", [(3, 64, 700), (90, 72, 5000), (601, 260, 1009)])
def test_entries_masked_by_the_lowest_fp32(ctx, T, d, vocab):
    H, W, t, stay = _masked("fp32", T, d, vocab, 1.0, torch.finfo(torch.float32).min)
    _against_the_rest(ctx, H, W, t, stay, "fp32", grad=True)


def test_fp32_operands_up_to_the_largest(ctx):
    """Products that are exact powers of two or the largest value itself, on either side: log-sum-exps of one entry."""
    T, d, vocab = 200, 8, 5000
    big = torch.finfo(torch.float32).max
    for of_h in (False, True):
        A, B = torch.zeros(T, d, device=DEV), torch.zeros(vocab, d, device=DEV)
        (A if of_h else B)[:, 0] = big
        (B if of_h else A)[:, 0] = 2.0 ** -120
        (B if of_h else A)[7, 0] = 2.0 ** -119
        want = float(big) * 2.0 ** -120                   # 256, to fp32
        lse = torch.empty(T, device=DEV)
        zo.zoact_ce_loss(ctx, A, B, ints(np.zeros(T)), lse=lse)
        torch.cuda.synchronize()
        assert ctx.device_status() == 0
        one = np.full(T, want + np.log(vocab))
        if of_h:                                         # entry 7 alone counts: 512 beside 256
            one[:] = 2 * want
        else:
            one[7] = 2 * want + np.log(vocab)
        within(lse, one, 2.0 ** -21 * one)


@pytest.mark.parametrize("dt,T,vocab", [("bf16", 40, 700), ("bf16", 1100, 900), ("fp16", 1100, 900), ("fp32", 8, 700),
                                        ("fp32", 300, 2000)])
def test_what_a_row_without_a_target_reaches(ctx, dt, T, vocab):
    """Its own log-sum-exp, which is finite where the row is, and nothing else."""
    d = 72
    H, W = rnd(1, T, d, dt=dt), rnd(2, vocab, d, std=0.2, dt=dt)
    t = np.random.default_rng(T).integers(0, vocab, T)
    t[[0, 2, T - 1]] = -1, -100, vocab                   # the last one is none of the vocabulary's
    none = torch.zeros(T, dtype=torch.bool, device=DEV)
    none[[0, 2, T - 1]] = True
    out = []
    for fill in (None, float("nan"), float("inf")):
        h = H.clone()
        if fill is not None:
            h[none] = fill
        dH, dW = torch.empty_like(h), torch.empty_like(W)
        loss, lse, mean = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
        zo.zoact_ce_grad(ctx, h, W, ints(t), dH=dH, dW=dW, loss=loss, lse=lse, mean=mean)
        torch.cuda.synchronize()
        assert ctx.device_status() == -1                 # the target that is not below the vocabulary
        lse2 = torch.empty_like(lse)
        zo.zoact_ce_loss(ctx, h, W, ints(t), lse=lse2)
        torch.cuda.synchronize()
        assert ctx.device_status() == -1
        assert torch.equal(lse[~none], lse2[~none])
        out.append((dH, dW, loss, mean, lse[~none]))
        if fill is None:
            wlse = ends.cross_entropy(n64(H), n64(W), np.zeros(T, dtype=int))[1]
            ez = (d + 8) * F * (np.abs(n64(H)) @ np.abs(n64(W)).T).max()
            within(lse, wlse, 2 * ez + 2.0 ** -20 + 4 * F * np.abs(wlse))
        else:
            assert not torch.isfinite(lse[none]).any()
    for other in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(out[0], other))
