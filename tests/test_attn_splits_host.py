"""Scratch of the token attention's backward where many rows meet few keys or the other way round: the shorter
side's partial gradients are not multiplied by the longer one's ranges."""
import pytest

from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)


@pytest.mark.parametrize("d", [32, 64])
@pytest.mark.parametrize("H, Hkv, Gq, Gk", [(8, 1, 1 << 17, 128), (64, 1, 1 << 14, 130), (64, 2, 1 << 15, 200)])
def test_many_rows_few_shared_keys(fs, H, Hkv, Gq, Gk, d):
    """What the call lays out of q and dout, rows and columns in two parts each, is 8 times q; its
    statistics are less than another half."""
    q = 4 * H * Gq * d
    assert fs.attn_workspace_bytes(fs.make_attn_shape(1, H, Gq, d, Hkv=Hkv, Gk=Gk), True) < 9 * q


@pytest.mark.parametrize("d", [32, 64])
def test_few_rows_many_keys(fs, d):
    """k and v: rows of both and columns of one, in two parts: 6 times k; dk and dv of one range of
    rows need no scratch."""
    k = 4 * (1 << 20) * d
    n = fs.attn_workspace_bytes(fs.make_attn_shape(1, 1, 128, d, Gk=1 << 20), True)
    assert n < 7 * k
