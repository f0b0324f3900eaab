"""Refusals of the token attention, on the host: every call here fails its checks before any
launch.  Addresses are fake and never read."""
import ctypes

import pytest
import torch

from test_abi_host import fs  # noqa: F401  (builds the library if it is not there)

P = ctypes.c_void_p
BASE, STEP = 1 << 32, 1 << 28


def addresses(n):
    return [BASE + i * STEP for i in range(n)]


def shape(fs, B=2, H=4, Hkv=2, Gq=40, Gk=50, d=32, mask=0, scale=0.1, cap=0.0):
    return fs.fs_attn_shape(B, H, Hkv, Gq, Gk, d, mask, scale, cap)


def mask(fs, **kw):
    m = fs.fs_attn_mask()
    for n, v in kw.items():
        setattr(m, n, v)
    return m


FWD = ["q", "k", "v", "out", "lse", "ws"]
BWD = ["q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv", "ws"]


def forward(fs, s, m=None, nbytes=1 << 40, **kw):
    a = {**dict(zip(FWD, addresses(6))), **kw}
    p = [P(a[n]) if a[n] else None for n in FWD]
    return fs._lib.fs_attn_fwd(ctypes.byref(s), *p[:3], None if m is None else ctypes.byref(m), *p[3:6], nbytes, None)


def backward(fs, s, m=None, nbytes=1 << 40, **kw):
    a = {**dict(zip(BWD, addresses(10))), **kw}
    p = [P(a[n]) if a[n] else None for n in BWD]
    return fs._lib.fs_attn_bwd(ctypes.byref(s), *p[:3], None if m is None else ctypes.byref(m), *p[3:10], nbytes, None)


@pytest.mark.parametrize("bad", [dict(B=0), dict(H=0), dict(Hkv=0), dict(Hkv=3), dict(Gq=0), dict(Gk=0), dict(Gk=-1),
                                 dict(d=0), dict(mask=2), dict(mask=1, Gq=51), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-44, scale=10.0),
                                 dict(B=1 << 40, H=1 << 20)])
def test_bad_shapes(fs, bad):
    s = shape(fs, **bad)
    assert forward(fs, s) == fs.FS_ERR_INVALID and backward(fs, s) == fs.FS_ERR_INVALID
    assert fs.attn_workspace_bytes(s) == 0 == fs.attn_workspace_bytes(s, True)


@pytest.mark.parametrize("far", [dict(d=48), dict(d=128), dict(B=20000), dict(Gk=(1 << 20) + 1),
                                 dict(Gq=(1 << 19) + 1, Gk=1 << 20)])
def test_unsupported_shapes(fs, far):
    s = shape(fs, **far)
    assert forward(fs, s) == fs.FS_ERR_UNSUPPORTED and backward(fs, s) == fs.FS_ERR_UNSUPPORTED
    assert fs.attn_workspace_bytes(s) == 0


def test_workspace(fs):
    for kw in (dict(), dict(Gq=1), dict(Gq=512, Gk=512, H=8, Hkv=8), dict(d=64), dict(Gq=4096, Gk=4096)):
        s = shape(fs, **kw)
        for call, bwd in ((forward, False), (backward, True)):
            n = fs.attn_workspace_bytes(s, bwd)
            assert n >= 256
            assert call(fs, s, nbytes=n - 1) == fs.FS_ERR_INVALID


def test_pointers(fs):
    s = shape(fs)
    qb, kb = 2 * 4 * 40 * 32 * 4, 2 * 2 * 50 * 32 * 4
    for names, call in ((FWD, forward), (BWD, backward)):
        at = dict(zip(names, addresses(len(names))))
        for n in names:
            assert call(fs, s, **{n: None}) == fs.FS_ERR_INVALID
            assert call(fs, s, **{n: at[n] + 8}) == fs.FS_ERR_INVALID
        outs = ["out", "lse"] if call is forward else ["dq", "dk", "dv"]
        for o in outs:
            for n in names:
                if n != o:  # an output over an input, the workspace or another output, or by its last bytes
                    assert call(fs, s, **{o: at[n]}) == fs.FS_ERR_INVALID
        assert call(fs, s, **{outs[0]: at["k"] + kb - 16}) == fs.FS_ERR_INVALID
        assert call(fs, s, **{outs[0]: at["q"] - qb + 16}) == fs.FS_ERR_INVALID


def test_masks(fs):
    a = addresses(20)[12:]
    for call in (forward, backward):
        for bad in (dict(slopes=a[0], pos_q=a[1]), dict(slopes=a[0], pos_k=a[1]), dict(pos_q=a[0], pos_k=a[1]),
                    dict(doc_q=a[0]), dict(doc_k=a[0]), dict(prefix=a[0]), dict(slopes=a[0] + 2),
                    dict(doc_q=a[0] + 1, doc_k=a[1])):
            assert call(fs, shape(fs), mask(fs, **bad)) == fs.FS_ERR_INVALID
        # an output over what a mask holds
        o = "out" if call is forward else "dq"
        for n in ("slopes", "prefix"):
            assert call(fs, shape(fs, mask=1), mask(fs, **{n: a[0]}), **{o: a[0]}) == fs.FS_ERR_INVALID
        assert call(fs, shape(fs), mask(fs, doc_q=a[0], doc_k=a[1]), **{o: a[1]}) == fs.FS_ERR_INVALID


def test_the_binding_checks_each_tensor(fs):
    s = fs.make_attn_shape(1, 2, 4, 16)
    q, lse, ws = torch.zeros(1, 2, 4, 16), torch.zeros(1, 2, 4), torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="q is on cpu"):
        fs.fs_attn_fwd(s, q, q, q, None, q, lse, ws)
    with pytest.raises(ValueError, match="q has 128 values of torch.bfloat16"):
        fs.fs_attn_fwd(s, q.bfloat16(), q, q, None, q, lse, ws)
    with pytest.raises(ValueError, match="q has 64 values"):
        fs.fs_attn_bwd(s, q[:, :1], q, q, None, q, lse, q, q, q, q, ws)
    with pytest.raises(ValueError, match="q is missing"):
        fs.fs_attn_fwd(s, None, q, q, None, q, lse, ws)
    assert fs.make_attn_shape(1, 2, 4, 16).scale == 0.25 and s.Hkv == 2 and s.Gk == 4
