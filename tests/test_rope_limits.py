"""Frequencies of the rotation at the ends of a double's range: those that are no number are refused, and nothing is written."""
import ctypes

import pytest

from paper_2607_01125_gb300 import _lib
from paper_2607_01125_gb300 import build as zbuild


@pytest.mark.parametrize("bad", [dict(scaling="linear", factor=5e-324), dict(scaling="parts", factor=5e-324),
                                 dict(rot=64, scaling="base", factor=1e-310, base=1.5)])   # base 1.5e-320, its power -62/64: 1e310
def test_frequencies_without_a_value_are_refused(bad):
    zbuild.build()
    with pytest.raises(_lib.ZoactError):
        _lib.rope(**{"rot": 4, **bad})
    r = _lib.zoact_rope(rot=-7, layout=-7)
    how = {"rot": 4, "factor": 1.0, "base": 10000.0, **bad}
    st = _lib.load().zoact_rope_init(ctypes.byref(r), how["rot"], 0, how["base"], _lib.ROPE_SCALING[how["scaling"]], how["factor"], 1.0, 4.0, 8192)
    assert st == -1 and r.rot == -7 and r.layout == -7 and not any(r.turns)


@pytest.mark.parametrize("good", [dict(scaling="linear", factor=1e-300), dict(scaling="linear", factor=1e300), dict(base=1e308),
                                  dict(rot=4, scaling="base", factor=1e-155, base=1.5),     # base 1.5e-310, its root 1e-155
                                  dict(base=1.0000001), dict(scaling="base", factor=1e-3), dict(scaling="parts", factor=1e300)])
def test_frequencies_at_the_ends_are_taken(good):
    zbuild.build()
    r = _lib.rope(**{"rot": 64, **good})
    assert r.rot == good.get("rot", 64) and all(0 <= t < 2 ** 64 for t in r.turns)
