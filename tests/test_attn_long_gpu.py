"""Token attention forward and backward at thousands of tokens, on tcgen05, against the fp64 oracle: long
ranges, several splits of either side, each head width (tests/_attn.py has the cases and derives the bounds)."""
import pytest

import _attn
from test_attn_paths_host import TCGEN05, paths

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size, what", [((1, 1, 1, 4096, 4096, 16), dict(prefix=1, cap=20.0)),
                                        ((1, 2, 1, 4096, 4096, 32), dict(prefix=1, bias="index")),
                                        ((1, 1, 1, 4096, 4096, 64), dict(docs=3, cap=30.0)),
                                        ((1, 1, 1, 4096, 4096, 64), dict(bias="place")),
                                        ((1, 1, 1, 130, 12000, 32), dict()), ((1, 1, 1, 130, 12000, 64), dict(docs=2)),
                                        ((1, 8, 1, 1300, 150, 32), dict(cap=5.0)), ((1, 8, 1, 1100, 400, 16), dict()),
                                        ((1, 8, 1, 1300, 150, 64), dict(bias="index"))],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else "-".join(v) or "plain")
def test_against_the_oracle(lib, size, what):
    assert paths(lib, size) == (TCGEN05, TCGEN05)
    _attn.check(lib, _attn.make(sum(size), *size, **what))
