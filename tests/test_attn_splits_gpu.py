"""Token attention where many rows share few keys: splits of the keys and of the rows apart, against the fp64
oracle (tests/_attn.py has the cases and derives the bounds)."""
import pytest

import _attn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [16, 32, 64])
@pytest.mark.parametrize("size", [(1, 8, 1, 256, 256), (1, 8, 1, 300, 130), (2, 16, 2, 100, 320), (1, 8, 1, 1000, 129),
                                  (1, 2, 1, 64, 2100)], ids=lambda s: "x".join(map(str, s)))
def test_shared_heads(lib, size, d):
    _attn.check(lib, _attn.make(sum(size) + d, *size, d, cap=4.0 if d == 32 else 0.0, docs=2 if size[1] == 16 else 0))


def test_shared_heads_under_the_prefix_mask(lib):
    _attn.check(lib, _attn.make(1, 1, 8, 1, 256, 330, 32, prefix=1, bias="index"))
