"""Caps far above every score: the scores as they are, to fp32's accuracy (tests/_attn.py derives the bounds)."""
import pytest

import _attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.18, 1e-3])
@pytest.mark.parametrize("cap", [1e30, 1e36, 1e38, 2e38, 3.4e38])
def test_huge_caps(lib, cap, scale):
    for H, G in ((2, 50), (4, 640)):
        c = _attn.make(G, 1, H, H, G, G, 32, cap=cap, docs=2)
        c["q"] *= 0.18 / scale  # scores of some units either way
        _attn.check(lib, {**c, "scale": scale})
