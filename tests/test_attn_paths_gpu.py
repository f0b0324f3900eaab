"""Token attention on both sides of each limit between warps and tcgen05, against the fp64 oracle
(tests/_attn.py has the cases and derives the bounds)."""
import pytest

import _attn
from test_attn_paths_host import NEIGHBOURS, paths

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size, forward, backward", NEIGHBOURS, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else None)
def test_both_sides_of_each_limit(lib, size, forward, backward):
    assert paths(lib, size) == (forward, backward)
    _attn.check(lib, _attn.make(sum(size), *size, bias="index" if size[3] == 360 else None))
