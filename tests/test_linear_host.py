"""Refusals of the linear maps and of dropout, on the host: every call here fails its checks
before any launch.  Addresses are fake and never read."""
import ctypes

import pytest
import torch

from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)

P = ctypes.c_void_p
FWD = ["x", "W", "bias", "act", "p", "rng", "res", "y", "pre"]
BWD = ["x", "W", "g", "act", "p", "rng", "pre", "dres", "dx", "dW", "dbias"]
OPTIONS = {"act": 2, "p": 0.5}


def base(names):
    at = {n: (1 << 30) + i * (1 << 24) for i, n in enumerate(names)}
    return {**at, **OPTIONS}


def raw(names, kw):
    return [kw[n] if n == "act" else ctypes.c_float(kw[n]) if n == "p" else P(kw[n]) for n in names]


def forward(fs, s, ws=1 << 40, nbytes=None, **kw):
    n = fs.linear_workspace_bytes(s) if nbytes is None else nbytes
    return fs._lib.fs_linear_fwd(ctypes.byref(s), *raw(FWD, {**base(FWD), **kw}), P(ws), n, None)


def backward(fs, s, ws=1 << 40, nbytes=None, **kw):
    n = fs.linear_workspace_bytes(s, True) if nbytes is None else nbytes
    return fs._lib.fs_linear_bwd(ctypes.byref(s), *raw(BWD, {**base(BWD), **kw}), 0, P(ws), n, None)


@pytest.mark.parametrize("bad", [(0, 8, 8, 0), (-1, 8, 8, 0), (4, 0, 8, 0), (4, 8, -2, 1), (4, 8, 8, 2), (1 << 40, 1, 2, 0),
                                 (1 << 39, 2, 1, 1)])
def test_bad_sizes(fs, bad):
    s = fs.fs_linear(*bad)
    assert forward(fs, s, nbytes=1 << 40) == fs.FS_ERR_INVALID
    assert backward(fs, s, nbytes=1 << 40) == fs.FS_ERR_INVALID
    assert fs.linear_workspace_bytes(s) == 0 and fs.linear_workspace_bytes(s, True) == 0
    assert fs.linear_path_for_shape(s) == -1


def test_too_many_channels(fs):
    for s in (fs.make_linear(4, 8193, 8), fs.make_linear(4, 8, 8193)):
        assert forward(fs, s, nbytes=1 << 40) == fs.FS_ERR_UNSUPPORTED
        assert backward(fs, s, nbytes=1 << 40) == fs.FS_ERR_UNSUPPORTED
        assert fs.linear_workspace_bytes(s) == 0 and fs.linear_path_for_shape(s, True) == -1
    assert fs.linear_workspace_bytes(fs.make_linear(4, 8192, 8192)) > 0


DROPS = [{"act": -1}, {"act": 4}, {"p": -0.1}, {"p": 1.0}, {"p": float("nan")}, {"p": float("inf")}, {"rng": None}]


@pytest.mark.parametrize("bad", DROPS)
def test_bad_activation_or_dropout(fs, bad):
    s = fs.make_linear(100, 64, 48)
    assert forward(fs, s, **bad) == fs.FS_ERR_INVALID
    assert backward(fs, s, **bad) == fs.FS_ERR_INVALID
    rows, kw = fs.make_rows(100, 64), {**base(FWD), **bad}
    for call, names in ((fs._lib.fs_dropout_fwd, ["x", "act", "p", "rng", "res", "y"]),
                        (fs._lib.fs_dropout_bwd, ["x", "act", "p", "rng", "pre", "y"])):
        assert call(ctypes.byref(rows), *raw(names, kw), None) == fs.FS_ERR_INVALID


def test_forward_pointers(fs):
    s, a = fs.make_linear(100, 64, 48), base(FWD)
    for n in ("x", "W", "y"):
        assert forward(fs, s, **{n: None}) == fs.FS_ERR_INVALID
    for n in FWD:
        if n not in OPTIONS:
            assert forward(fs, s, **{n: a[n] + 8}) == fs.FS_ERR_INVALID
    assert forward(fs, s, y=a["x"]) == fs.FS_ERR_INVALID
    assert forward(fs, s, y=a["res"] + 16) == fs.FS_ERR_INVALID          # in place only byte for byte
    assert forward(fs, s, y=a["W"] + 64 * 48 * 4 - 16) == fs.FS_ERR_INVALID
    assert forward(fs, s, y=a["rng"]) == fs.FS_ERR_INVALID
    assert forward(fs, s, pre=a["res"]) == fs.FS_ERR_INVALID
    assert forward(fs, s, pre=a["y"]) == fs.FS_ERR_INVALID
    assert forward(fs, s, pre=a["res"], y=a["res"]) == fs.FS_ERR_INVALID
    for ws in (None, a["x"], a["y"], a["res"], (1 << 40) + 4):
        assert forward(fs, s, ws=ws) == fs.FS_ERR_INVALID
    assert forward(fs, s, nbytes=fs.linear_workspace_bytes(s) - 1) == fs.FS_ERR_INVALID


def test_backward_pointers(fs):
    s, a = fs.make_linear(100, 64, 48), base(BWD)
    for n in ("x", "W", "g", "pre"):
        assert backward(fs, s, **{n: None}) == fs.FS_ERR_INVALID
    assert backward(fs, s, dW=None) == fs.FS_ERR_INVALID                 # dbias alone
    assert backward(fs, s, dx=None) == fs.FS_ERR_INVALID                 # dres for no dx
    assert backward(fs, s, dx=None, dW=None, dbias=None, dres=None) == fs.FS_ERR_INVALID
    for n in BWD:
        if n not in OPTIONS:
            assert backward(fs, s, **{n: a[n] + 8}) == fs.FS_ERR_INVALID
    for out in ("dx", "dW", "dbias"):
        for other in ("x", "W", "g", "pre", "dW" if out == "dx" else "dx"):
            assert backward(fs, s, **{out: a[other]}) == fs.FS_ERR_INVALID
    assert backward(fs, s, dx=a["dres"] + 16) == fs.FS_ERR_INVALID
    assert backward(fs, s, dW=a["dres"]) == fs.FS_ERR_INVALID
    for ws in (None, a["g"], a["dres"], a["dx"]):
        assert backward(fs, s, ws=ws) == fs.FS_ERR_INVALID
    assert backward(fs, s, nbytes=fs.linear_workspace_bytes(s, True) - 1) == fs.FS_ERR_INVALID


def test_dropout_pointers(fs):
    rows, a = fs.make_rows(100, 40), base(FWD)
    calls = ((fs._lib.fs_dropout_fwd, ["x", "act", "p", "rng", "res", "y"], "res"),
             (fs._lib.fs_dropout_bwd, ["x", "act", "p", "rng", "pre", "y"], "pre"))
    for call, names, third in calls:
        def go(rows=rows, **kw):
            return call(ctypes.byref(rows), *raw(names, {**a, **kw}), None)

        for n in ("x", "y"):
            assert go(**{n: None}) == fs.FS_ERR_INVALID
        for n in names:
            if n not in OPTIONS:
                assert go(**{n: a[n] + 4}) == fs.FS_ERR_INVALID
        assert go(y=a["x"] + 16) == fs.FS_ERR_INVALID
        assert go(y=a[third] + 16) == fs.FS_ERR_INVALID
        assert go(y=a["rng"]) == fs.FS_ERR_INVALID
        assert go(rows=fs.fs_rows(0, 40, 0)) == fs.FS_ERR_INVALID
        assert go(rows=fs.make_rows(4, 8193)) == fs.FS_ERR_UNSUPPORTED
    assert fs._lib.fs_dropout_bwd(ctypes.byref(rows), *raw(calls[1][1], {**a, "pre": None}), None) == fs.FS_ERR_INVALID


def test_the_binding_checks_each_tensor(fs):
    s, rows = fs.make_linear(6, 8, 4), fs.make_rows(6, 8)
    x, W, y, ws = torch.zeros(6, 8), torch.zeros(4, 8), torch.zeros(6, 4), torch.zeros(1 << 16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="x is on cpu"):
        fs.fs_linear_fwd(s, x, W, None, fs.FS_ACT_NONE, 0.0, None, None, y, None, ws)
    with pytest.raises(ValueError, match="x has 48 values of torch.bfloat16"):
        fs.fs_linear_fwd(s, x.bfloat16(), W, None, fs.FS_ACT_NONE, 0.0, None, None, y, None, ws)
    with pytest.raises(ValueError, match="x must be contiguous"):
        fs.fs_linear_fwd(s, torch.zeros(8, 6).T, W, None, fs.FS_ACT_NONE, 0.0, None, None, y, None, ws)
    with pytest.raises(ValueError, match="x has 24 values"):
        fs.fs_dropout_fwd(rows, y, fs.FS_ACT_NONE, 0.0, None, None, x)
    with pytest.raises(ValueError, match="dy is missing"):
        fs.fs_dropout_bwd(rows, None, fs.FS_ACT_NONE, 0.0, None, None, x)
    with pytest.raises(ValueError):
        fs.make_linear(6, 8, 4, torch.float16)
    r = fs.dropout_rng((1 << 64) - 1, 5, "cpu")
    assert r.tolist() == [-1, 5] and r.dtype is torch.int64


def test_the_path_goes_by_the_products_size(fs):
    """Both sides of each limit: 2^24 products for bf16, 2^27 for fp32; more than eight rows."""
    for dtype, rows in ((fs.FS_BF16, 256), (fs.FS_F32, 2048)):
        for backward in (False, True):
            assert fs.linear_path_for_shape(fs.make_linear(rows, 256, 256, dtype), backward) == 1
            assert fs.linear_path_for_shape(fs.make_linear(rows - 1, 256, 256, dtype), backward) == 0
    assert fs.linear_path_for_shape(fs.make_linear(8, 8192, 8192, fs.FS_BF16)) == 0
    assert fs.linear_path_for_shape(fs.make_linear(9, 8192, 8192, fs.FS_BF16)) == 1
    assert fs.linear_path_for_shape(fs.make_linear(1 << 20, 3, 256, fs.FS_BF16)) == 1   # coordinates in, a few results out
    assert fs.linear_path_for_shape(fs.make_linear(1 << 20, 256, 1, fs.FS_BF16)) == 1
    assert fs.linear_path_for_shape(fs.make_linear((1 << 31) - 512, 16, 16, fs.FS_BF16)) == 0  # past TMA's coordinates
