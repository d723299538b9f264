"""Stacks whose mixer is attention over packed sequences (ZOStep.pack): against the fp64 oracle, and the properties of packing --
a sequence sees itself only, a token nothing behind it -- in ZO steps on tokens.

Tolerances: fp32 within 2e-5 of the outputs' root mean square (sums of up to 512 terms in a dozen products, 2^-24 each, and
logits' errors that shares multiply).  16-bit: an error of a score is an error of its share times the share, so roundings of q and k
grow with the spread of the scores (here 4: by about that much in each decoder, 4 2^-8 / sqrt(12) of every rounding of the first).
How much, the oracle says: with the activations rounded where the graph stores them it makes the same errors up to the
draw, so the root mean squares over 10^4 outputs agree to a few percent; twice the oracle's own distance bounds the GPU's.
"""
import numpy as np
import pytest
import torch

import paper_2607_01125_gb300 as zo
from oracle import decoder, graphs
from oracle.layers import STORE_ROUNDING, rms_norm, silu
from paper_2607_01125_gb300.model import AdaptedLinear, TokenStep, ZOStep, calibrate_bases
from synth import normal

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
D, KV, HID, HEAD = 256, 128, 512, 64
SHAPES = {"llama": [("q", D, D), ("k", D, KV), ("v", D, KV), ("o", D, D), ("gate", D, HID), ("up", D, HID), ("down", HID, D)],
          "opt": [("q", D, D), ("k", D, D), ("v", D, D), ("o", D, D), ("fc1", D, HID), ("fc2", HID, D)]}


def n64(t):
    return t.detach().double().cpu().numpy()


def stack(ctx, dt, T, n_dec=2, n_queries=None, r=8):
    """A llama-like stack, or (fp32, which has no gated call) an OPT-like one."""
    kind = "opt" if dt == "fp32" else "llama"
    lins, off, bases = [], 0, {}
    for L in range(n_dec):
        for i, (name, d_in, d_out) in enumerate(SHAPES[kind]):
            lid = 7 * L + i
            key = (L, "qkv") if name in "qkv" else (L, "gu") if name in ("gate", "up") else (L, name)
            U = bases.setdefault(key, torch.linalg.qr(normal((d_in, r), 50 + lid, DEV))[0].contiguous())
            # q and k larger than the rest, so that shares differ
            std = (2.0 if name in ("q", "k") else 1.0) * d_in ** -0.5
            lins.append(AdaptedLinear(f"{L}.{name}", normal((d_out, d_in), lid, DEV, std=std).to(TYPES[dt]), U, lid, off, r))
            off += (d_out * r + 3) // 4 * 4
    s = ZOStep(ctx, kind, lins, T, dt, eps=1e-2, lr=1e-3, n_heads=4, n_kv_heads=2, head_dim=HEAD, n_queries=n_queries)
    s.C.copy_(normal((s.C.numel(),), 99, DEV, std=0.05))
    return s


def oracle(s, x, seed, query, lengths, rope, blocks, store="fp64"):
    """The same graph with attention for its mixer; activations rounded to `store` where the graph stores them."""
    rnd = STORE_ROUNDING[store]
    layer = {l.name: dict(W=n64(l.W), U=n64(l.U), C=n64(s.C[l.offset:l.offset + l.d_out * l.r]).reshape(l.d_out, l.r),
                          layer_id=l.layer_id) for l in s.linears}
    T, nb = s.T, s.nb
    spans = [tuple(int(v) for v in row + np.array([b * T, 0, b * T, 0])) for b in range(nb)
             for row in zo.attention_spans(lengths).numpy()]
    pos = np.concatenate([np.arange(n) for n in lengths] + [np.zeros(T - sum(lengths), dtype=int)])
    h, shared = x, True

    def lin(name, X, sh=False):
        return graphs.layer_forward(layer[name], X, s.eps, seed, query, T, sh, blocks)

    for L in range(len(s.groups)):
        a = rnd(rms_norm(h))
        q, k, v = (rnd(lin(f"{L}.{n}", a, shared)).reshape(nb * T, -1, HEAD) for n in "qkv")
        shared = False
        if rope is not None:
            q, k = (rnd(decoder.rope(t, pos, rope, "half")) for t in (q, k))
        mix = rnd(np.nan_to_num(decoder.attention(q, k, v, spans, True, HEAD ** -0.5)[0])).reshape(nb * T, -1)
        b = rnd(rms_norm(rnd(lin(f"{L}.o", mix))))
        if s.kind == "llama":
            h = rnd(lin(f"{L}.down", rnd(rms_norm(rnd(silu(lin(f"{L}.gate", b)) * lin(f"{L}.up", b))))))
        else:
            h = rnd(lin(f"{L}.fc2", rnd(rms_norm(rnd(np.maximum(lin(f"{L}.fc1", b), 0.0))))))
    return h


@pytest.mark.parametrize("dt,n_queries,T", [("fp32", None, 40), ("bf16", None, 40), ("bf16", None, 150), ("bf16", 2, 110), ("fp16", None, 150)])
@pytest.mark.parametrize("turned", [True, False])
def test_packed_stack_against_the_oracle(dt, n_queries, T, turned):
    ctx = zo.Context(0)
    s = stack(ctx, dt, T, n_queries=n_queries)
    lengths = [T // 2, 1, 0, T // 3]                                     # rows behind the last sequence
    rope = zo.rope(HEAD, base=500.0) if turned else None
    x = normal((T, D), 7, DEV).to(TYPES[dt])
    s.pack(lengths, rope)
    Y = s.forward(x, 3, 5)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    blocks = None if n_queries is None else s.points(5)
    args = (s, n64(x), 3, 5, lengths, decoder.frequencies(HEAD, 500.0) if turned else None, blocks)
    want = oracle(*args)
    rows = np.concatenate([np.arange(sum(lengths)) + b * T for b in range(s.nb)])

    def distance(y):
        return np.sqrt(((y[rows] - want[rows]) ** 2).mean())

    bound = 2e-5 * np.sqrt((want[rows] ** 2).mean()) if dt == "fp32" else 2 * distance(oracle(*args, store=dt))
    assert distance(n64(Y)) <= bound, (distance(n64(Y)), bound)
    assert np.abs(n64(Y)).max() < 1e4                                    # and nothing wild behind them
    ctx.close()


@pytest.mark.parametrize("dt,T", [("fp32", 40), ("bf16", 160)])
def test_sequences_and_later_tokens_are_not_seen(dt, T):
    ctx = zo.Context(0)
    s = stack(ctx, dt, T)
    table = normal((50, D), 1, DEV).to(TYPES[dt])
    model = TokenStep(s, table, gain=torch.ones(D, device=DEV), bias=torch.zeros(D, device=DEV))
    n = T // 2
    s.pack([n, T - n - 3], zo.rope(HEAD))
    ids = torch.randint(0, 50, (T,), generator=torch.Generator(DEV).manual_seed(1), device=DEV)
    first = model.forward(ids, 1, 2).clone()
    other = ids.clone()
    other[n] = (other[n] + 7) % 50                                       # the second sequence's first token
    second = model.forward(other, 1, 2).clone()
    for b in range(2):
        assert torch.equal(first[b * T:b * T + n], second[b * T:b * T + n])
        assert not torch.equal(first[b * T + T - 4], second[b * T + T - 4])
    other = ids.clone()
    other[n - 1] = (other[n - 1] + 7) % 50                               # the first one's last token
    second = model.forward(other, 1, 2).clone()
    for b in range(2):
        assert torch.equal(first[b * T:b * T + n - 1], second[b * T:b * T + n - 1])
        assert not torch.equal(first[b * T + n - 1], second[b * T + n - 1])
        assert torch.equal(first[b * T + n:b * T + T - 3], second[b * T + n:b * T + T - 3])
    targets = torch.where(torch.arange(T, device=DEV) < T - 3, ids.roll(-1), torch.full_like(ids, -100))
    C = s.C.clone()
    out = model.step(ids, targets, 1, seed=1, query=2).clone()
    torch.cuda.synchronize()
    assert ctx.device_status() == 0 and torch.isfinite(out).all() and not torch.equal(C, s.C)
    ctx.close()


def test_mixers_come_and_go():
    """pack(None) gives the synthetic mixer back, with the results it had; other packings make other results."""
    ctx = zo.Context(0)
    s = stack(ctx, "bf16", 150)
    x = normal((150, D), 7, DEV).to(torch.bfloat16)
    before = s.forward(x, 1, 1).clone()
    s.pack([150])
    whole = s.forward(x, 1, 1).clone()
    s.pack([75, 75])
    halves = s.forward(x, 1, 1).clone()
    s.pack([150])
    assert torch.equal(s.forward(x, 1, 1), whole) and not torch.equal(whole, before)
    assert torch.equal(halves[:75], whole[:75]) and not torch.equal(halves[75:150], whole[75:150])
    s.pack(None)
    assert torch.equal(s.forward(x, 1, 1), before)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for lengths in ([151], [100, 51], [-1]):
        with pytest.raises(ValueError):
            s.pack(lengths)
    lin = [AdaptedLinear(n, torch.zeros(256, 256, device=DEV), torch.zeros(256, 8, device=DEV), i, 2048 * i, 8)
           for i, n in enumerate(("l1", "l2"))]
    with pytest.raises(ValueError):
        ZOStep(ctx, "toy", lin, 8, "fp32").pack([8])
    ctx.close()


def test_bases_calibrated_with_attention():
    """A calibration pass of a packed stack: every basis is orthonormal, and that of o the one of attention's outputs."""
    ctx = zo.Context(0)
    s = stack(ctx, "bf16", 300, n_dec=1)
    s.C.zero_()
    s.pack([200, 100], zo.rope(HEAD))
    x = normal((300, D), 7, DEV).to(torch.bfloat16)
    calibrate_bases(ctx, s, x, 8)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for l in s.linears:
        U = n64(l.U)
        assert np.abs(U.T @ U - np.eye(8)).max() < 1e-4
    X = n64(s._bufs["attn"][:300])
    vals = np.linalg.eigvalsh(X.T @ X)
    U = n64(s.by_name["0.o"].U)
    assert np.trace(U.T @ X.T @ X @ U) >= 0.99 * vals[-8:].sum()
    ctx.close()
