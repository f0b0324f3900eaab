"""One to sixteen rows through wide maps: which kernels they run by, and that each gives the right results."""
import pytest

import _linear as t
from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)


def test_dx_goes_by_the_products_size(fs):
    """From one row on; the kernel for few rows is the forward's."""
    for dtype, rows in ((fs.FS_BF16, 1), (fs.FS_BF16, 8), (fs.FS_F32, 2), (fs.FS_F32, 8)):
        assert fs.linear_path_for_shape(fs.make_linear(rows, 8192, 8192, dtype), True) == 1
    assert fs.linear_path_for_shape(fs.make_linear(1, 8192, 8192, fs.FS_F32), True) == 0
    assert fs.linear_path_for_shape(fs.make_linear(3, 4096, 1024, fs.FS_BF16), True) == 0
    assert fs.linear_path_for_shape(fs.make_linear(4, 4096, 1024, fs.FS_BF16), True) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N, dtype", [(1, 8192, 2100, "bf16"), (2, 4097, 2051, "bf16"), (8, 2046, 1030, "bf16"), (4, 1024, 4096, "bf16"),
                                            (7, 4096, 4098, "f32"), (8, 4099, 4101, "f32"), (9, 2048, 1000, "bf16")])
def test_backward(lib, R, K, N, dtype):
    assert lib.linear_path_for_shape(lib.make_linear(R, K, N, t.DTYPES[dtype]), True) == (R * K * N >= (1 << 24 if dtype == "bf16" else 1 << 27))
    t.check_backward(lib, R, K, N, dtype, seed=R)
    t.check_backward(lib, R, K, N, dtype, "gelu", 0.25, dres=True, inplace=True, want_dw=False, seed=R + 1)


@pytest.mark.gpu
def test_narrow_forwards_go_by_rows_and_terms(lib):
    """Fewer columns than 16 an SM: both sides of 8192 rows times terms, 16,384 where the other path are multiply-adds."""
    assert lib.linear_path_for_shape(lib.make_linear(4, 2048, 2048, lib.FS_BF16)) == 0
    assert lib.linear_path_for_shape(lib.make_linear(5, 2048, 2048, lib.FS_BF16)) == 1
    assert lib.linear_path_for_shape(lib.make_linear(8, 2048, 8192, lib.FS_BF16)) == 0
    assert lib.linear_path_for_shape(lib.make_linear(8, 4096, 2048, lib.FS_F32)) == 0
    # a split sum has parts in the workspace
    size = lambda R, K, N: lib.linear_workspace_bytes(lib.make_linear(R, K, N, lib.FS_F32))  # noqa: E731
    assert size(4, 4096, 1024) == 256 and size(5, 4096, 1024) > 256


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N, dtype", [(8, 4096, 1024, "bf16"), (3, 8192, 1024, "bf16"), (4, 8192, 256, "bf16"), (7, 8189, 250, "bf16"), (5, 2049, 2047, "bf16"),
                                            (5, 4096, 1024, "f32"), (8, 8191, 130, "f32"), (2, 8192, 1024, "bf16"), (8, 1024, 2048, "f32"), (1, 8192, 16, "f32"),
                                            (8, 2048, 2500, "bf16")])
def test_forward(lib, R, K, N, dtype):
    t.check_forward(lib, R, K, N, dtype, seed=R)
    t.check_forward(lib, R, K, N, dtype, "gelu", 0.25, res=True, pre=True, seed=R + 1)
    t.check_forward(lib, R, K, N, dtype, "relu", 0.1, res=True, inplace=True, seed=R + 2)
