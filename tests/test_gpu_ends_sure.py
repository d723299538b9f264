"""Cross entropy of rows that the model is nearly sure of: with a target's share of 1 - S the loss is S (to S^2), the gradient by the
target's logit -S, and the gradient by the hidden state the difference of the other entries' and S times the target's
weights.  All of them keep S's own digits, whether the other entries lie in the target's 128 of the vocabulary or not.

Tolerances: S is a sum of exponentials of differences of two logits, each a sum of d products in fp32 (F = 2^-24), so it errs by
2 ez + 2^-20 of itself; G is rounded to the operands' type (bf16 2^-8, fp16 2^-11 and its kept logits 2^-12; fp32: three parts),
fp16's in multiples of 2^-24 of a scale of 2^15; the results to theirs.
"""
import numpy as np
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


def within(got, want, tol):
    got = got.double()
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= tol).all(), float(((got - want).abs() / tol.clamp(min=1e-300)).max())


# rows on the MMA's N side and (20011 entries) on its M side; fp32 as it is and (from 300 rows on) in parts
@pytest.mark.parametrize("dt,T,vocab", [("bf16", 3, 130), ("bf16", 40, 640), ("bf16", 1200, 1009), ("bf16", 601, 20011),
                                        ("fp16", 3, 130), ("fp16", 1100, 1009), ("fp16", 601, 20011), ("fp32", 3, 130), ("fp32", 300, 640), ("fp32", 1500, 20011)])
def test_rows_that_are_nearly_sure(ctx, dt, T, vocab):
    d = 256
    g = torch.Generator(DEV).manual_seed(T)
    W = (torch.randn(vocab, d, generator=g, device=DEV) / 16).to(TYPES[dt])
    t = torch.randperm(vocab, generator=g, device=DEV).repeat(T // vocab + 1)[:T]
    w = W.double()
    lead = 14 + 10 * torch.rand(T, 1, generator=g, device=DEV).double()     # of the target's logit: S from 1e-3 to 1e-8
    H = (lead * w[t] / w[t].square().sum(dim=1, keepdim=True)).to(TYPES[dt])
    h = H.double()
    z = h @ w.t()
    at = torch.arange(T, device=DEV)
    other = torch.exp(z - z[at, t][:, None])
    other[at, t] = 0
    S = other.sum(dim=1)                                # the others' shares beside the target's, S / (1 + S) of all
    loss = torch.log1p(S)
    assert float(S.median()) < 1e-3 and float(S.min()) < 5e-6
    ez = ((d + 8) * F * (h.abs() @ w.abs().t())).max(dim=1).values
    rel = 2 * ez + 2.0 ** -20 + 8 * F
    got, mean = torch.empty(T, device=DEV), torch.empty(1, dtype=torch.float64, device=DEV)
    zo.zoact_ce_loss(ctx, H, W, t, loss=got, mean=mean)
    dH, dW, loss2 = torch.empty_like(H), torch.empty(vocab, d, device=DEV), torch.empty(T, device=DEV)
    zo.zoact_ce_grad(ctx, H, W, t, dH=dH, dW=dW, loss=loss2)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    within(got, loss, rel * loss)
    assert torch.equal(got, loss2)
    within(mean, loss.mean()[None], (rel * loss).mean()[None])

    G = other / (1 + S)[:, None]
    G[at, t] = -S / (1 + S)
    ug = 2.0 ** -21 if dt == "fp32" else 1.01 * UNIT[dt] + 2.0 ** -11
    eg = (ug + rel[:, None]) * G.abs() + (2.0 ** -40 if dt == "fp16" else 0)
    th = (eg @ w.abs() + (vocab + 8) * F * (G.abs() @ w.abs())) / T
    tw = (eg.t() @ h.abs() + (T + 8) * F * (G.abs().t() @ h.abs())) / T
    wh, ww = G @ w / T, G.t() @ h / T
    within(dH, wh, th + UNIT[dt] * (wh.abs() + th) + TINY[dt])
    within(dW, ww, tw + F * ww.abs())
