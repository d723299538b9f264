"""The fp64 oracle of a language model's two ends: its gradients against differences, its edge cases by their definition."""
import numpy as np
import pytest

from oracle import ends


def _num_grad(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        g[i] = (up - f()) / (2 * h)
        x[i] = keep
    return g


def test_cross_entropy_gradient_is_that_of_its_mean():
    rng = np.random.default_rng(1)
    H, W = rng.standard_normal((6, 5)), rng.standard_normal((9, 5))
    t = np.array([3, -100, 0, 8, 3, -1])
    f = lambda: 2.5 * ends.cross_entropy(H, W, t)[2][0]
    dH, dW = ends.cross_entropy_grad(H, W, t, 2.5)
    assert np.abs(dH - _num_grad(f, H)).max() < 1e-8 and np.abs(dW - _num_grad(f, W)).max() < 1e-8
    assert (dH[1] == 0).all() and (dH[5] == 0).all()


def test_cross_entropy_of_uncounted_rows_and_large_logits():
    H, W = np.array([[1000.0, 0.0], [0.0, 0.0]]), np.array([[1.0, 0.0], [-1.0, 0.0], [0.0, 1.0]])
    loss, lse, mean = ends.cross_entropy(H, W, [0, 1])
    assert loss[0] == 0.0 and lse[0] == 1000.0 and abs(loss[1] - np.log(3)) < 1e-15
    loss, _, mean = ends.cross_entropy(H, W, [-1, -1])
    assert (loss == 0).all() and mean[0] == 0.0
    loss, _, mean = ends.cross_entropy(np.concatenate([H, H + 1.0]), W, [1, -1], n_blocks=2)
    assert loss[1] == loss[3] == 0.0 and mean[0] == loss[0] and mean[1] == loss[2]
    assert np.allclose(ends.pair(mean, loss, [1, -1], 0.5), [loss[0], loss[2], loss[0] - loss[2], loss[0] - loss[2]])


@pytest.mark.parametrize("with_gain", [True, False])
def test_layer_norm_gradient_is_that_of_its_output(with_gain):
    rng = np.random.default_rng(2)
    X, c = rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    g, b = (rng.standard_normal(7), rng.standard_normal(7)) if with_gain else (None, None)
    Y, m, s = ends.layer_norm(X, g, b, 1e-3)
    dX, dg, db = ends.layer_norm_grad(c, X, g, m, s)
    f = lambda: (c * ends.layer_norm(X, g, b, 1e-3)[0]).sum()
    assert np.abs(dX - _num_grad(f, X)).max() < 1e-7
    if with_gain:
        assert np.abs(dg - _num_grad(f, g)).max() < 1e-7 and np.abs(db - _num_grad(f, b)).max() < 1e-7


def test_embedding_gradient_is_that_of_its_rows():
    rng = np.random.default_rng(3)
    E, ids, c = rng.standard_normal((6, 4)), np.array([2, -100, 5, 2, 0]), rng.standard_normal((5, 4))
    assert (ends.embed(E, ids, 3.0)[1] == 0).all()
    f = lambda: (c * ends.embed(E, ids, 3.0)).sum()
    dE = ends.embed_grad(c, ids, 6, 3.0)
    assert np.abs(dE - _num_grad(f, E)).max() < 1e-7
    assert np.allclose(ends.embed_grad(c, ids, 6, 3.0, start=E), E + dE)


def test_the_forward_passes_are_those_of_torch():
    import torch
    import torch.nn.functional as tf
    rng = np.random.default_rng(4)
    H, W, X = rng.standard_normal((7, 5)), rng.standard_normal((11, 5)), rng.standard_normal((4, 9))
    g, b, t = rng.standard_normal(9), rng.standard_normal(9), np.array([0, 10, -100, 3, 3, -100, 7])
    T = torch.as_tensor
    loss, lse, mean = ends.cross_entropy(H, W, t)
    z = T(H) @ T(W).T
    assert np.allclose(loss, tf.cross_entropy(z, T(t), reduction="none", ignore_index=-100), rtol=1e-13, atol=1e-13)
    assert np.allclose(mean[0], tf.cross_entropy(z, T(t), ignore_index=-100), rtol=1e-13)
    assert np.allclose(lse, torch.logsumexp(z, 1), rtol=1e-13)
    assert np.allclose(ends.layer_norm(X, g, b, 1e-5)[0], tf.layer_norm(T(X), (9,), T(g), T(b), 1e-5), rtol=1e-12, atol=1e-13)
    ids = np.array([4, 0, 10, 4])
    assert np.allclose(ends.embed(W, ids, 0.5), 0.5 * tf.embedding(T(ids), T(W)))
