"""The fp64 oracle of rotary positions and attention: properties, a worked case, and its gradients against differences.  The host
part of the rotation (frequencies as fractions of a turn) and refusals that need no GPU."""
import ctypes
import math

import numpy as np
import pytest

from oracle import decoder
from paper_2607_01125_gb300 import _lib
from paper_2607_01125_gb300 import build as zbuild


def test_attention_of_two_keys_by_hand():
    q, k = np.array([[[2.0]], [[1.0]]]), np.array([[[1.0]], [[0.0]]])
    v = np.array([[[10.0]], [[20.0]]])
    O, lse = decoder.attention(q, k, v, [(0, 2, 0, 2)], True, 0.5)
    e = math.exp(0.5)
    assert np.allclose(O[:, 0, 0], [10.0, (10 * e + 20) / (e + 1)], rtol=1e-14)
    assert np.allclose(lse[:, 0], [1.0, math.log(e + 1)], rtol=1e-14)


def test_rows_that_see_no_key():
    q, k = np.ones((5, 2, 3)), np.ones((2, 1, 3))
    O, lse = decoder.attention(q, k, k, [(0, 4, 0, 2)], True, 1.0)
    assert (O[:2] == 0).all() and (lse[:2] == -np.inf).all() and np.allclose(O[2:4], 1.0) and np.isnan(O[4]).all()


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradient_against_differences(causal):
    rng = np.random.default_rng(1)
    q, k, v, G = (rng.standard_normal(s) for s in ((7, 4, 5), (9, 2, 5), (9, 2, 5), (7, 4, 5)))
    spans, scale = [(0, 2, 0, 4), (2, 1, 4, 0), (3, 4, 4, 3)], 0.4

    def loss(*x):
        return np.nansum(decoder.attention(*x, spans, causal, scale)[0] * G)

    O, lse = decoder.attention(q, k, v, spans, causal, scale)
    grads = decoder.attention_grad(G, q, k, v, O, lse, spans, causal, scale)
    for n, x in enumerate((q, k, v)):
        for _ in range(12):
            at = tuple(rng.integers(0, s) for s in x.shape)
            args = [q.copy(), k.copy(), v.copy()]
            args[n][at] += 1e-5
            up = loss(*args)
            args[n][at] -= 2e-5
            slope = (up - loss(*args)) / 2e-5
            got = grads[n][at]
            assert abs(slope - (0.0 if np.isnan(got) else got)) < 1e-7


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_keeps_products_of_one_distance(layout):
    rng = np.random.default_rng(2)
    f = decoder.frequencies(6, 100.0)
    a, b = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
    dots = [(decoder.rope(a, [p + 3], f, layout) * decoder.rope(b, [p], f, layout)).sum() for p in (0, 11, 500)]
    assert np.allclose(dots, dots[0])
    back = decoder.rope(decoder.rope(a, [77], f, layout), [77], f, layout, inverse=True)
    assert np.allclose(back, a)


@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (256, 1e6)])
def test_frequencies_in_turns(rot, base, scaling):
    zbuild.build()
    how = dict(factor=8.0, low=1.0, high=4.0, original=8192)
    r = _lib.rope(rot, base=base, scaling=scaling, **how)
    f = decoder.frequencies(rot, base, scaling, **how)
    got = np.array([r.turns[i] for i in range(rot // 2)], dtype=np.float64) * 2.0 ** -64 * 2 * math.pi
    # a power and a handful of roundings in fp64; the turns' own step is 2^-64
    assert np.abs(got - f).max() <= 1e-13 and (np.abs(got - f) <= 1e-13 * f + 1e-18).all()
    assert all(r.turns[i] == 0 for i in range(rot // 2, _lib.ROPE_MAX // 2))
    if scaling == "base" and rot > 2:
        assert np.isclose(got[-1], decoder.frequencies(rot, base)[-1] / 8.0)


@pytest.mark.parametrize("bad", [dict(rot=0), dict(rot=3), dict(rot=258), dict(base=1.0), dict(base=float("nan")),
                                 dict(scaling="linear", factor=0.0), dict(scaling="parts", factor=8.0, low=4.0, high=4.0),
                                 dict(scaling="parts", factor=8.0, original=0), dict(scaling="base", factor=float("inf"))])
def test_rope_refusals(bad):
    zbuild.build()
    with pytest.raises(_lib.ZoactError):
        _lib.rope(**{"rot": 64, **bad})
    with pytest.raises(ValueError):
        _lib.rope(64, layout="other")


def test_calls_without_a_context_are_refused():
    zbuild.build()
    lib, s = _lib.load(), _lib.attention_shape(4, 4, 1, 2, 2, 8)
    buf = ctypes.create_string_buffer(1024)
    p = ctypes.addressof(buf)
    assert lib.zoact_attention_plan_bytes(None, ctypes.byref(s), 0) == -1
    assert lib.zoact_attention_plan(None, ctypes.byref(s), p, 1, 0, p) == -1
    assert lib.zoact_attention(None, ctypes.byref(s), p, p, 16, p, 16, p, 16, 0, 1.0, p, 16, None) == -1
    assert lib.zoact_rope_apply(None, p, 0, 1, 1, 2, 2, p, 1, 1, ctypes.byref(_lib.rope(2)), 0, p, 2) == -1


def test_struct_layouts():
    assert ctypes.sizeof(_lib.zoact_attention_shape) == 40 and _lib.zoact_attention_shape.n_seq.offset == 16
    assert ctypes.sizeof(_lib.zoact_rope) == 8 + 8 * 128 and _lib.zoact_rope.turns.offset == 8


def test_spans_of_packed_sequences():
    assert _lib.attention_spans([3, 0, 2]).tolist() == [[0, 3, 0, 3], [3, 0, 3, 0], [3, 2, 3, 2]]
    assert _lib.attention_spans([1, 1], [7, 5], [0, 16]).tolist() == [[0, 1, 0, 7], [1, 1, 16, 5]]
    assert _lib.attention_spans([]).shape == (0, 4)
    with pytest.raises(ValueError):
        _lib.attention_spans([1], [1, 2])
