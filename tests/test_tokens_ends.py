"""Ends of the ranges that the operators of long videos take, as far as no GPU is needed."""
import math

import pytest

from paper_2510_05367_amd import binding as lcb
from paper_2510_05367_amd import tokens


@pytest.mark.parametrize("scaling,dim,factor", [("base", 4, 1e-200), ("base", 4, 1e200), ("base", 128, 1e305), ("linear", 64, 1e-320), ("linear", 64, 1e-30),
                                                ("parts", 64, 1e-310), ("base", 8, 1e-60)])
def test_rope_tables_hold_numbers(scaling, dim, factor):
    """A factor that takes base or frequencies out of the range of 64 bits would turn by angles that are no numbers, or by none."""
    with pytest.raises(lcb.LcError, match="factor") as e:
        tokens.make_rope(dim, scaling=scaling, factor=factor, orig_len=4096)
    assert e.value.status == lcb.LC_ERR_SHAPE


@pytest.mark.parametrize("scaling,dim,factor", [("base", 4, 1e100), ("base", 128, 1e-3), ("base", 2, 1e300), ("linear", 64, 1e-9), ("linear", 64, 1e300), ("parts", 64, 1e-9)])
def test_rope_tables_of_wide_factors(scaling, dim, factor):
    t = tokens.make_rope(dim, scaling=scaling, factor=factor, orig_len=4096)
    for i in range(dim // 2):
        base = 1e4 * factor ** (dim / (dim - 2)) if scaling == "base" and dim > 2 else 1e4
        w = base ** (-2 * i / dim)
        if scaling == "linear":
            w /= factor
        if scaling == "parts":
            keep = min(max((4096 * w / (2 * math.pi) - 1) / 31, 0), 1)
            w *= keep + (1 - keep) / factor
        assert t.turns[i] == pytest.approx(w / (2 * math.pi), rel=1e-12)
