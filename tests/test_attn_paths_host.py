"""Which kernels a token attention call runs by (fs_attn_path_for_shape): the rule's limits, and the shapes of
the GPU tests that are meant for the one or the other."""
import pytest

from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)

WARPS, TCGEN05 = 0, 1
# B, H, Hkv, Gq, Gk, d; forward, backward
NEIGHBOURS = [
    # rows of a unit
    *[((1, 12, 12, rows, 1000, d), path, path) for d in (16, 32, 64) for rows, path in ((127, WARPS), (128, TCGEN05))],
    ((1, 48, 12, 31, 1100, 32), WARPS, WARPS), ((1, 48, 12, 32, 1100, 32), TCGEN05, TCGEN05),  # shared heads together
    # keys
    *[((1, 12, 12, 1000, keys, d), path, path) for d in (32, 64) for keys, path in ((127, WARPS), (128, TCGEN05))],
    ((1, 11, 11, 360, 383, 16), WARPS, TCGEN05), ((1, 11, 11, 360, 384, 16), TCGEN05, TCGEN05),
    ((1, 17, 17, 256, 255, 16), WARPS, WARPS), ((1, 17, 17, 256, 256, 16), WARPS, TCGEN05),
    # pairs: 1.5 million forward; 1.1 million backward, 0.7 at d = 64
    *[((1, 1, 1, 1224, 1225, d), WARPS, TCGEN05) for d in (16, 32, 64)],
    *[((1, 1, 1, 1225, 1225, d), TCGEN05, TCGEN05) for d in (16, 32, 64)],
    *[((1, 1, 1, 1048, 1049, d), WARPS, WARPS if d < 64 else TCGEN05) for d in (16, 32, 64)],
    *[((1, 1, 1, 1049, 1049, d), WARPS, TCGEN05) for d in (16, 32, 64)],
    ((1, 1, 1, 836, 837, 64), WARPS, WARPS), ((1, 1, 1, 837, 837, 64), WARPS, TCGEN05),
]
# those of tests/test_attn_gpu.py that are for tcgen05
LARGE = [(1, 16, 4, 100, 1000), (1, 8, 8, 440, 440), (1, 8, 8, 600, 330), (12, 8, 8, 128, 128), (2, 8, 2, 129, 760),
         (1, 1, 1, 1300, 1301), (1, 16, 1, 33, 3000)]


def paths(fs, size):
    B, H, Hkv, Gq, Gk, d = size
    s = fs.make_attn_shape(B, H, Gq, d, Hkv=Hkv, Gk=Gk)
    return fs.attn_path_for_shape(s), fs.attn_path_for_shape(s, True)


@pytest.mark.parametrize("size, forward, backward", NEIGHBOURS, ids=lambda s: "x".join(map(str, s)) if isinstance(s, tuple) else None)
def test_both_sides_of_each_limit(fs, size, forward, backward):
    assert paths(fs, size) == (forward, backward)


def test_the_large_shapes_of_the_gpu_tests(fs):
    for d in (16, 32, 64):
        for size in LARGE:
            few = d == 16 and (size[3:] == (128, 128) or size[3:] == (600, 330))
            assert paths(fs, (*size, d)) == (WARPS if few else TCGEN05, WARPS if few and size[4] == 128 else TCGEN05)


def test_small_shapes(fs):
    for size in ((1, 1, 1, 1, 1, 32), (1, 8, 8, 32, 32, 32), (2, 8, 2, 1, 700, 32), (1, 8, 2, 130, 130, 32),
                 (2, 2, 2, 256, 256, 32), (1, 2, 2, 600, 129, 32), (4, 8, 2, 1, 4096, 32)):
        assert paths(fs, size) == (WARPS, WARPS)


def test_none_for_a_bad_shape(fs):
    assert paths(fs, (1, 4, 3, 10, 10, 32)) == (-1, -1)   # invalid
    assert paths(fs, (1, 4, 4, 10, 10, 48)) == (-1, -1)   # unsupported
