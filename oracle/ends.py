"""The two ends of a language model in fp64, from their formulas: embedding rows by token id, layer norm, and the cross
entropy of a head over the vocabulary, each with its gradient.

A negative id or target is no token: a zero row, no gradient, a loss of 0 that is not counted in the mean.
"""
import numpy as np


def embed(E, ids, scale):
    Y = np.zeros((len(ids), E.shape[1]))
    for t, v in enumerate(ids):
        if v >= 0:
            Y[t] = scale * E[v]
    return Y


def embed_grad(dY, ids, vocab, scale, start=None):
    dE = np.zeros((vocab, dY.shape[1])) if start is None else np.array(start, dtype=np.float64)
    for t, v in enumerate(ids):
        if v >= 0:
            dE[v] += scale * dY[t]
    return dE


def layer_norm(X, gain, bias, eps):
    """(Y, mean, rstd); gain and bias may be None."""
    m = X.mean(axis=1)
    s = 1.0 / np.sqrt(((X - m[:, None]) ** 2).mean(axis=1) + eps)
    Y = (X - m[:, None]) * s[:, None]
    Y = Y if gain is None else Y * gain
    return Y if bias is None else Y + bias, m, s


def layer_norm_grad(dY, X, gain, mean, rstd):
    """(dX, dgain, dbias) for the statistics as given."""
    xh = (X - mean[:, None]) * rstd[:, None]
    u = dY if gain is None else dY * gain
    dX = rstd[:, None] * (u - u.mean(axis=1, keepdims=True) - xh * (u * xh).mean(axis=1, keepdims=True))
    return dX, (dY * xh).sum(axis=0), dY.sum(axis=0)


def cross_entropy(H, W, targets, n_blocks=1):
    """(loss [rows], lse [rows], mean [n_blocks]) for H [n_blocks T, d], W [vocab, d], targets [T]."""
    z = H @ W.T
    top = z.max(axis=1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    t = np.tile(np.asarray(targets), n_blocks)
    loss = np.where(t >= 0, lse - z[np.arange(len(t)), np.maximum(t, 0)], 0.0)
    count = max(1, int((np.asarray(targets) >= 0).sum()))
    return loss, lse, loss.reshape(n_blocks, -1).sum(axis=1) / count


def cross_entropy_grad(H, W, targets, grad_scale=1.0):
    """(dH, dW) of grad_scale times the mean loss."""
    t = np.asarray(targets)
    z = H @ W.T
    G = np.exp(z - z.max(axis=1, keepdims=True))
    G /= G.sum(axis=1, keepdims=True)
    G[np.arange(len(t)), np.maximum(t, 0)] -= 1.0
    G *= (t >= 0)[:, None] * grad_scale / max(1, int((t >= 0).sum()))
    return G @ W, G.T @ H


def pair(L, loss, targets, eps):
    """{L+, L-, D, a} from the blocks' means and the rows' losses (D from the rows' differences)."""
    T = len(targets)
    count = max(1, int((np.asarray(targets) >= 0).sum()))
    D = (loss[:T] - loss[T:]).sum() / count
    return np.array([L[0], L[1], D, D / (2 * eps)])
