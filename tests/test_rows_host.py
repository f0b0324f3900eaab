"""Refusals of the layer norm and the 8-bit checkpoint, on the host: every call here fails its
checks before any launch.  Addresses are fake and never read."""
import ctypes

import pytest
import torch

from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)

P = ctypes.c_void_p


def addresses(n, step=1 << 24):
    return [(1 << 30) + i * step for i in range(n)]


def norm_fwd(fs, rows, args, eps=1e-5):
    x, res, gamma, beta, out_sum, y, mean, rstd, q8, e8 = args
    return fs._lib.fs_norm_fwd(ctypes.byref(rows), P(x), P(res), P(gamma), P(beta), eps, P(out_sum), P(y), P(mean),
                               P(rstd), P(q8), P(e8), None)


def norm_bwd(fs, rows, args, ws=1 << 40, nbytes=None):
    n = fs.norm_workspace_bytes(rows) if nbytes is None else nbytes
    return fs._lib.fs_norm_bwd(ctypes.byref(rows), *[P(a) for a in args], 0, P(ws), n, None)


BAD_ROWS = [(0, 32, 0), (-1, 32, 0), (4, 0, 0), (4, -3, 0), (4, 32, 5), (1 << 40, 2, 0)]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_bad_rows(fs, bad):
    a, rows = addresses(11), fs.fs_rows(*bad)
    assert norm_fwd(fs, rows, a[:10]) == fs.FS_ERR_INVALID
    assert norm_bwd(fs, rows, [a[0], None, None] + a[3:11], nbytes=1 << 40) == fs.FS_ERR_INVALID
    assert fs._lib.fs_ckpt_pack(ctypes.byref(rows), P(a[0]), P(a[1]), P(a[2]), None) == fs.FS_ERR_INVALID
    assert fs._lib.fs_ckpt_unpack(ctypes.byref(rows), P(a[0]), P(a[1]), P(a[2]), None) == fs.FS_ERR_INVALID
    assert fs.norm_workspace_bytes(rows) == 0


def test_too_many_channels(fs):
    a, rows = addresses(11), fs.make_rows(4, 8193)
    assert norm_fwd(fs, rows, a[:10]) == fs.FS_ERR_UNSUPPORTED
    assert norm_bwd(fs, rows, [a[0], None, None] + a[3:11], nbytes=1 << 40) == fs.FS_ERR_UNSUPPORTED
    assert fs._lib.fs_ckpt_pack(ctypes.byref(rows), P(a[0]), P(a[1]), P(a[2]), None) == fs.FS_ERR_UNSUPPORTED
    assert fs.norm_workspace_bytes(rows) == 0 and fs.norm_workspace_bytes(fs.make_rows(4, 8192)) > 0


def test_norm_fwd_pointers(fs):
    rows, a = fs.make_rows(100, 64), addresses(10)
    names = ["x", "res", "gamma", "beta", "sum", "y", "mean", "rstd", "q8", "e8"]

    def call(**kw):
        return norm_fwd(fs, rows, [kw.get(n, v) for n, v in zip(names, a)])

    for n in ("x", "y"):
        assert call(**{n: None}) == fs.FS_ERR_INVALID
    for n, v in zip(names, a):
        assert call(**{n: v + 4}) == fs.FS_ERR_INVALID
    assert call(res=None) == fs.FS_ERR_INVALID               # sum without a residual
    assert call(q8=None) == fs.FS_ERR_INVALID                # half a checkpoint
    assert call(e8=None) == fs.FS_ERR_INVALID
    assert call(y=a[0]) == fs.FS_ERR_INVALID                 # y over x
    assert call(sum=a[0] + 16) == fs.FS_ERR_INVALID          # in place only byte for byte
    assert call(sum=a[5] + 16) == fs.FS_ERR_INVALID          # two outputs
    assert call(q8=a[1] + 100 * 64 * 4 - 16) == fs.FS_ERR_INVALID
    assert call(rstd=a[6]) == fs.FS_ERR_INVALID
    for eps in (-1e-5, float("nan"), float("inf")):
        assert norm_fwd(fs, rows, a, eps) == fs.FS_ERR_INVALID


def test_norm_bwd_pointers(fs):
    rows, a = fs.make_rows(100, 64), addresses(11)
    names = ["v", "q8", "e8", "gamma", "mean", "rstd", "dy", "dres", "dv", "dgamma", "dbeta"]

    def call(ws=1 << 40, nbytes=None, **kw):
        base = dict(zip(names, a), q8=None, e8=None)
        return norm_bwd(fs, rows, [{**base, **kw}[n] for n in names], ws, nbytes)

    for n in ("v", "mean", "rstd", "dy", "dv"):
        assert call(**{n: None}) == fs.FS_ERR_INVALID
    for n, v in zip(names, a):
        if n not in ("q8", "e8"):
            assert call(**{n: v + 8}) == fs.FS_ERR_INVALID
    assert call(q8=a[1], e8=a[2]) == fs.FS_ERR_INVALID       # rows and their checkpoint
    assert call(v=None, q8=a[1]) == fs.FS_ERR_INVALID
    assert call(dgamma=None) == fs.FS_ERR_INVALID            # one parameter gradient alone
    assert call(dv=a[0]) == fs.FS_ERR_INVALID                # over v
    assert call(dv=a[6] + 16) == fs.FS_ERR_INVALID
    assert call(dgamma=a[6]) == fs.FS_ERR_INVALID
    assert call(ws=None, nbytes=1 << 30) == fs.FS_ERR_INVALID
    assert call(ws=a[0]) == fs.FS_ERR_INVALID
    assert call(nbytes=fs.norm_workspace_bytes(rows) - 1) == fs.FS_ERR_INVALID


def test_checkpoint_pointers(fs):
    rows, (x, q8, e8) = fs.make_rows(100, 40), addresses(3)
    for call, args in ((fs._lib.fs_ckpt_pack, (x, q8, e8)), (fs._lib.fs_ckpt_unpack, (q8, e8, x))):
        for i in range(3):
            for bad in (None, args[i] + 2):
                assert call(ctypes.byref(rows), *[P(bad if j == i else v) for j, v in enumerate(args)],
                            None) == fs.FS_ERR_INVALID
        over = [x if v in (q8, x) else v for v in args]
        assert call(ctypes.byref(rows), *[P(v) for v in over], None) == fs.FS_ERR_INVALID


def test_the_binding_checks_each_tensor(fs):
    rows = fs.make_rows(6, 8)
    x, q8, e8 = torch.zeros(6, 8), torch.zeros(6, 8, dtype=torch.int8), torch.zeros(6, 1, dtype=torch.uint8)
    with pytest.raises(ValueError, match="x is on cpu"):
        fs.fs_ckpt_pack(rows, x, q8, e8)
    with pytest.raises(ValueError, match="x has 48 values of torch.float64"):
        fs.fs_ckpt_pack(rows, x.double(), q8, e8)
    with pytest.raises(ValueError, match="x has 40 values"):
        fs.fs_ckpt_pack(rows, x[:5], q8, e8)
    with pytest.raises(ValueError, match="x must be contiguous"):
        fs.fs_ckpt_pack(rows, torch.zeros(8, 6).T, q8, e8)
    with pytest.raises(ValueError, match="x is missing"):
        fs.fs_norm_fwd(rows, None, None, None, None, 1e-5, None, x, None, None)
    with pytest.raises(ValueError):
        fs.make_rows(6, 8, torch.float16)
    assert fs.rows_of(torch.zeros(2, 3, 4, 8), C=32).rows == 6
