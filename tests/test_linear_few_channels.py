"""fp32 maps of few channels: which path they run by, and that both sides of each limit are right."""
import pytest

import _linear as t
from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)

ROWS = 1 << 20


def test_paths(fs):
    forward = lambda K, N, dtype=fs.FS_F32: fs.linear_path_for_shape(fs.make_linear(ROWS, K, N, dtype))  # noqa: E731
    dx = lambda K, N, dtype=fs.FS_F32: fs.linear_path_for_shape(fs.make_linear(ROWS, K, N, dtype), True)  # noqa: E731
    assert [forward(32, 64), forward(33, 64), forward(32, 65)] == [0, 1, 1]
    assert [forward(3, 256), forward(15, 1024), forward(16, 256)] == [0, 0, 1]
    assert [dx(64, 32), dx(64, 33), dx(65, 32)] == [0, 1, 1]     # g's channels are the terms
    assert dx(256, 3) == 1
    for K, N in ((2, 64), (3, 256), (32, 64)):
        assert forward(K, N, fs.FS_BF16) == 1 and dx(N, K, fs.FS_BF16) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N", [(140000, 3, 330), (70000, 32, 64), (70000, 33, 64), (70000, 32, 66), (140000, 64, 17), (40000, 64, 64), (40000, 64, 65),
                                     (140000, 16, 65), (36000, 63, 62), (140000, 1, 1024)])
def test_both_sides(lib, R, K, N):
    t.check_forward(lib, R, K, N, "f32", seed=R)
    t.check_forward(lib, R, K, N, "f32", "gelu", 0.25, res=True, pre=True, seed=R + 1)
    t.check_backward(lib, R, K, N, "f32", seed=R)
    t.check_backward(lib, R, K, N, "f32", "silu", 0.1, dres=True, accumulate=True, seed=R + 1)
