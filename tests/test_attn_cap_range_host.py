"""Scales and caps whose products with log2(e) leave fp32's range are refused (on the host; addresses are fake)."""
import pytest

from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)
from test_attn_host import backward, forward, shape


@pytest.mark.parametrize("bad", [dict(scale=3e38), dict(scale=-3e38), dict(scale=4.0, cap=3e38), dict(scale=-2.4e38),
                                 dict(scale=3.0, cap=2.4e38)])
def test_refused(fs, bad):
    s = shape(fs, **bad)
    assert forward(fs, s) == fs.FS_ERR_INVALID and backward(fs, s) == fs.FS_ERR_INVALID
    assert fs.attn_workspace_bytes(s) == 0


@pytest.mark.parametrize("good", [dict(scale=2e38), dict(scale=0.2, cap=3.4e38), dict(scale=2.0, cap=2.4e38), dict(scale=0.0, cap=3.4e38),
                                  dict(scale=4.0, cap=2e38), dict(scale=3e38, cap=2.0)])
def test_taken(fs, good):
    assert fs.attn_workspace_bytes(shape(fs, **good)) > 0
