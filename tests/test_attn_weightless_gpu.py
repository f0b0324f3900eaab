"""A visible key whose weight underflows to 0 adds nothing, whatever its value holds: the results are those
without it (tests/_attn.py derives the bounds), and its own gradients are 0."""
import numpy as np
import pytest

import _attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("d", [16, 32, 64])
@pytest.mark.parametrize("H, G", [(2, 60), (4, 640)])
def test_a_key_without_weight(lib, H, G, d, bad):
    c = _attn.make(H + d, 1, H, H, G, G, d)
    c["q"] = np.abs(c["q"]) + np.float32(0.5)
    c["k"][:, :, 5] = -400.0  # scores of -400 sqrt(d) / 2 and less, the others' are some tens at most
    c["v"][:, :, 5] = bad
    got = _attn.run(lib, c)
    rest = {**c, "Gk": G - 1, **{n: np.delete(c[n], 5, 2) for n in ("k", "v")}}
    mine = {n: np.delete(t, 5, 2) if n in ("dk", "dv") else t for n, t in got.items()}
    _attn.check(lib, rest, mine)
    assert (got["dk"][:, :, 5] == 0).all() and (got["dv"][:, :, 5] == 0).all()
