"""Inside a decoder in fp64, from the formulas: rotary positions, and attention over packed sequences with its gradient.

Arrays are [rows, heads, head_dim]; spans a list of (first query row, queries, first key row, keys).  A query i of a causal
sequence sees the keys j <= i + (keys - queries); a row that sees none has an output of 0 and a log-sum-exp of -inf.
"""
import math

import numpy as np


def frequencies(rot, base, scaling="none", factor=1.0, low=1.0, high=4.0, original=8192):
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = np.array([base ** (-2 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        t = original * f / (2 * math.pi)
        for i in range(len(f)):
            if t[i] < low:
                f[i] /= factor
            elif t[i] <= high:
                s = (t[i] - low) / (high - low)
                f[i] *= s + (1 - s) / factor
    return f


def rope(x, positions, f, layout, inverse=False):
    """x [rows, heads, head_dim], positions [n] with rows a multiple of n."""
    y = np.array(x, dtype=np.float64)
    h = len(f)
    n = len(positions)
    for r in range(x.shape[0]):
        angle = float(positions[r % n]) * f * (-1 if inverse else 1)
        c, s = np.cos(angle), np.sin(angle)
        at = (slice(0, h), slice(h, 2 * h)) if layout == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
        a, b = x[r][:, at[0]], x[r][:, at[1]]
        y[r][:, at[0]], y[r][:, at[1]] = a * c - b * s, a * s + b * c
    return y


def seen(nq, nk, causal):
    i, j = np.arange(nq)[:, None], np.arange(nk)[None, :]
    return j <= i + (nk - nq) if causal else np.ones((nq, nk), dtype=bool)


def _sequences(q, k, spans, causal):
    for q0, nq, k0, nk in spans:
        for h in range(q.shape[1]):
            yield slice(q0, q0 + nq), slice(k0, k0 + nk), h, h // (q.shape[1] // k.shape[1]), seen(nq, nk, causal)


def attention(q, k, v, spans, causal, scale, size=False):
    """(O, lse) with NaN in the rows of no sequence; with size (O, lse, sum_j p_j |v_j|, largest sum of |q k| scale,
    sum_j |v_j|) for error bounds."""
    O = np.full(q.shape, np.nan)
    lse = np.full(q.shape[:2], np.nan)
    A, z, V = np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan), np.full(q.shape, np.nan)
    for rq, rk, h, g, m in _sequences(q, k, spans, causal):
        s = np.where(m, q[rq, h] @ k[rk, g].T * scale, -np.inf)
        top = s.max(axis=1, initial=-np.inf)
        p = np.exp(s - np.where(np.isfinite(top), top, 0.0)[:, None])
        l = p.sum(axis=1)
        with np.errstate(divide="ignore"):
            lse[rq, h] = top + np.log(l)
        p = p / np.where(l > 0, l, 1.0)[:, None]
        O[rq, h] = p @ v[rk, g]
        if size:
            A[rq, h] = p @ np.abs(v[rk, g])
            V[rq, h] = m @ np.abs(v[rk, g])
            z[rq, h] = np.where(m, np.abs(q[rq, h]) @ np.abs(k[rk, g]).T * scale, 0.0).max(axis=1, initial=0.0)
    return (O, lse, A, z, V) if size else (O, lse)


def attention_grad(dO, q, k, v, O, lse, spans, causal, scale, error=None):
    """(dq, dk, dv) for the O and lse as given, NaN in rows of no sequence.  With error = (relative error of a share, its
    factor of the sums of |q k| scale, relative error of dP and delta by their sums of magnitudes, rounding of P and dS, absolute
    rounding of both, relative error of the last sums) also bounds of the three."""
    out = [np.full(x.shape, np.nan) for x in (q, k, v)]
    tol = [np.full(x.shape, np.nan) for x in (q, k, v)]
    for rq, _, h, _, _ in _sequences(q, k, spans, causal):
        out[0][rq, h] = tol[0][rq, h] = 0.0
    for _, rk, _, g, _ in _sequences(q, k, spans, causal):
        for x in (out[1], out[2], tol[1], tol[2]):
            x[rk, g] = 0.0
    for rq, rk, h, g, m in _sequences(q, k, spans, causal):
        Q, K, V, G = q[rq, h], k[rk, g], v[rk, g], dO[rq, h]
        with np.errstate(invalid="ignore", over="ignore"):
            p = np.where(m, np.exp(Q @ K.T * scale - lse[rq, h][:, None]), 0.0)
        dp, delta = G @ V.T, (G * O[rq, h]).sum(axis=1)[:, None]
        ds = p * (dp - delta)
        out[0][rq, h] = ds @ K * scale
        out[1][rk, g] += ds.T @ Q * scale
        out[2][rk, g] += p.T @ G
        if error is not None:
            ep, ez, ed, u, tiny, es = error
            rel = ep + ez * (np.abs(Q) @ np.abs(K).T * scale)
            size = np.abs(G) @ np.abs(V).T + (np.abs(G) * np.abs(O[rq, h])).sum(axis=1)[:, None]
            e = np.abs(ds) * (rel + u + es) + p * ed * size + tiny * m
            tol[0][rq, h] += e @ np.abs(K) * scale
            tol[1][rk, g] += e.T @ np.abs(Q) * scale
            tol[2][rk, g] += (p * (rel + u + es) + tiny * m).T @ np.abs(G)
    return (*out, *tol) if error is not None else tuple(out)
