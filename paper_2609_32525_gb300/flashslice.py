"""Python binding of libflashslice.so (include/flashslice.h): argument marshalling only.

Every function named fs_* here calls the C entry point of the same name with
the device pointers of torch tensors and the current CUDA stream, and raises
FlashSliceError on a non-FS_OK status.  All compute happens in the library's
CUDA kernels; there is no fallback of any kind.  Importing this module loads
the library and fails loudly if it has not been built
(`python -m paper_2609_32525_gb300.build`).

Tensor conventions (see the header for the full contract):
  x_mid, fx, out, dout, dx_mid, dfx : [B,N,H,d] float32 or bfloat16, contiguous
  W_slice [H,d,G], bias [H,G], tau [H], M [H,G,G]            float32
  tokens, tokens_mixed, d_tokens*  [B,H,G,d], wsum [B,H,G], lse [B,H,N]  float32
"""
from __future__ import annotations

import ctypes
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libflashslice.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2609_32525_gb300.build` "
                      "(the library has no CPU fallback)")
_lib = ctypes.CDLL(_LIB_PATH)

FS_OK, FS_ERR_INVALID, FS_ERR_UNSUPPORTED, FS_ERR_CUDA, FS_ERR_TIMEOUT, FS_ERR_BAD_TAU, FS_ERR_SCRATCH_TOO_SMALL = range(7)
FS_NOALLOC_SCRATCH_BYTES = 16 << 20
FS_F32, FS_BF16 = 0, 1
FS_DOT_BF16, FS_DOT_BF16X2 = 0, 1
FS_MASK_NONE, FS_MASK_PREFIX = 0, 1
FS_ACT_NONE, FS_ACT_RELU, FS_ACT_GELU, FS_ACT_SILU = range(4)
FS_OP_SLICE_FWD, FS_OP_DESLICE_FWD, FS_OP_DESLICE_BWD, FS_OP_SLICE_BWD, FS_OP_STATS, FS_OP_COUPLING_BWD = range(6)

EXPORTED = ("fs_workspace_bytes", "fs_slice_fwd", "fs_slice_finalize", "fs_mix", "fs_deslice_fwd",
            "fs_deslice_bwd", "fs_mix_bwd", "fs_slice_bwd", "fs_device_status", "fs_status_string",
            "fs_path_for_shape", "fs_backward_path_for_shape", "fs_forward_launch_count", "fs_backward_launch_count",
            "fs_slice_fwd_noalloc", "fs_slice_fwd_lse", "fs_mix_channels", "fs_mix_channels_bwd", "fs_mix_channels_bwd_add", "fs_stats",
            "fs_coupling_bwd", "fs_coupling_bwd_launch_count", "fs_norm_fwd", "fs_norm_bwd",
            "fs_norm_workspace_bytes", "fs_ckpt_pack", "fs_ckpt_unpack", "fs_attn_fwd", "fs_attn_bwd",
            "fs_attn_workspace_bytes", "fs_attn_path_for_shape", "fs_linear_fwd", "fs_linear_bwd",
            "fs_linear_workspace_bytes", "fs_linear_path_for_shape", "fs_dropout_fwd", "fs_dropout_bwd")


class fs_shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("N", ctypes.c_int64), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("G", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("dot", ctypes.c_int32)]


class fs_rows(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class fs_linear(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("Cin", ctypes.c_int32), ("Cout", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class fs_attn_shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64)] + [(n, ctypes.c_int32) for n in ("H", "Hkv", "Gq", "Gk", "d", "mask")] + [
        ("scale", ctypes.c_float), ("cap", ctypes.c_float)]


class fs_attn_mask(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("slopes", "pos_q", "pos_k", "doc_q", "doc_k", "prefix")]


class FlashSliceError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__(f"{fn}: {_lib.fs_status_string(status).decode()}")


_P = ctypes.c_void_p
_S = ctypes.POINTER(fs_shape)
_I = ctypes.c_int
_Z = ctypes.c_size_t
_F = ctypes.c_float
_R = ctypes.POINTER(fs_rows)
_A = ctypes.POINTER(fs_attn_shape)
_M = ctypes.POINTER(fs_attn_mask)
_L = ctypes.POINTER(fs_linear)
_sig = {
    "fs_workspace_bytes": (_Z, [_S, _I]),
    "fs_slice_fwd": (_I, [_S, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _Z, _P]),
    "fs_slice_fwd_lse": (_I, [_S, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _Z, _P]),
    "fs_slice_finalize": (_I, [_S, _P, _P, _P]),
    "fs_stats": (_I, [_S, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "fs_mix_channels": (_I, [_S, _P, _P, _P, _P]),
    "fs_mix_channels_bwd": (_I, [_S, _P, _P, _P, _P, _P, _P]),
    "fs_mix_channels_bwd_add": (_I, [_S, _P, _P, _P, _P, _P, _P]),
    "fs_mix": (_I, [_S, _P, _P, _P, _P]),
    "fs_deslice_fwd": (_I, [_S, _P, _P, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "fs_deslice_bwd": (_I, [_S, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _Z, _P]),
    "fs_mix_bwd": (_I, [_S, _P, _P, _P, _P, _P, _P]),
    "fs_slice_bwd": (_I, [_S, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I, _P, _Z, _P]),
    "fs_device_status": (_I, [_P, _P]),
    "fs_status_string": (ctypes.c_char_p, [_I]),
    "fs_path_for_shape": (_I, [_S]),
    "fs_backward_path_for_shape": (_I, [_S]),
    "fs_forward_launch_count": (_I, [_S]),
    "fs_backward_launch_count": (_I, [_S, _I]),
    "fs_coupling_bwd_launch_count": (_I, [_S, _I]),
    "fs_coupling_bwd": (_I, [_S] + [_P] * 11 + [_P] * 8 + [_I, _P, _Z, _P]),
    "fs_attn_fwd": (_I, [_A, _P, _P, _P, _M, _P, _P, _P, _Z, _P]),
    "fs_attn_bwd": (_I, [_A, _P, _P, _P, _M, _P, _P, _P, _P, _P, _P, _P, _Z, _P]),
    "fs_attn_workspace_bytes": (_Z, [_A, _I]),
    "fs_attn_path_for_shape": (_I, [_A, _I]),
    "fs_norm_fwd": (_I, [_R] + [_P] * 4 + [_F] + [_P] * 7),
    "fs_norm_bwd": (_I, [_R] + [_P] * 11 + [_I, _P, _Z, _P]),
    "fs_norm_workspace_bytes": (_Z, [_R]),
    "fs_ckpt_pack": (_I, [_R, _P, _P, _P, _P]),
    "fs_ckpt_unpack": (_I, [_R, _P, _P, _P, _P]),
    "fs_linear_fwd": (_I, [_L, _P, _P, _P, _I, _F, _P, _P, _P, _P, _P, _Z, _P]),
    "fs_linear_bwd": (_I, [_L, _P, _P, _P, _I, _F] + [_P] * 6 + [_I, _P, _Z, _P]),
    "fs_linear_workspace_bytes": (_Z, [_L, _I]),
    "fs_linear_path_for_shape": (_I, [_L, _I]),
    "fs_dropout_fwd": (_I, [_R, _P, _I, _F, _P, _P, _P, _P]),
    "fs_dropout_bwd": (_I, [_R, _P, _I, _F, _P, _P, _P, _P]),
    "fs_slice_fwd_noalloc": (_I, [_S, _P, _P, _P, _P, _P, _P, _P, _P, _I, ctypes.POINTER(_P), _P]),
}
for _name, (_res, _args) in _sig.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def make_shape(B, N, H, d, G, dtype=FS_F32, eps=1e-5, dot=None) -> fs_shape:
    """dot: FS_DOT_BF16 (default) or FS_DOT_BF16X2 (see the header)."""
    if isinstance(dtype, torch.dtype):
        dtype = FS_BF16 if dtype == torch.bfloat16 else FS_F32
    return fs_shape(int(B), int(N), int(H), int(d), int(G), int(dtype), float(eps),
                    int(FS_DOT_BF16 if dot is None else dot))


def shape_of(x_mid: torch.Tensor, G: int, eps: float = 1e-5, dot=None) -> fs_shape:
    B, N, H, d = x_mid.shape
    return make_shape(B, N, H, d, G, x_mid.dtype, eps, dot)


def _ptr(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("flashslice tensors must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _check(fn, st):
    if st != FS_OK:
        raise FlashSliceError(fn, st)


def workspace_bytes(shape: fs_shape, op: int) -> int:
    return int(_lib.fs_workspace_bytes(ctypes.byref(shape), op))


def workspace(shape: fs_shape, op: int, device="cuda") -> torch.Tensor:
    """Scratch for one op, allocated through torch (the library never allocates).
    Its status word starts at FS_OK, so a scratch no call has used yet reads clean."""
    n = max(16, workspace_bytes(shape, op))
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    ws[:16].zero_()
    return ws


def path_for_shape(shape: fs_shape) -> int:
    return int(_lib.fs_path_for_shape(ctypes.byref(shape)))


def backward_path_for_shape(shape: fs_shape) -> int:
    return int(_lib.fs_backward_path_for_shape(ctypes.byref(shape)))


def forward_launch_count(shape: fs_shape) -> int:
    return int(_lib.fs_forward_launch_count(ctypes.byref(shape)))


def backward_launch_count(shape: fs_shape, lse_given: bool = True) -> int:
    return int(_lib.fs_backward_launch_count(ctypes.byref(shape), int(bool(lse_given))))


def coupling_bwd_launch_count(shape: fs_shape, lse_given: bool = True) -> int:
    return int(_lib.fs_coupling_bwd_launch_count(ctypes.byref(shape), int(bool(lse_given))))


def status_string(st: int) -> str:
    return _lib.fs_status_string(st).decode()


def fs_slice_fwd(shape, x_mid, fx, W_slice, bias, tau, tokens, wsum, lse, finalize, ws, stream=None):
    st = _lib.fs_slice_fwd(ctypes.byref(shape), _ptr(x_mid), _ptr(fx), _ptr(W_slice), _ptr(bias), _ptr(tau),
                           _ptr(tokens), _ptr(wsum), _ptr(lse), int(bool(finalize)), _ptr(ws), ws.numel(),
                           _stream(stream))
    _check("fs_slice_fwd", st)


def fs_stats(shape, x_mid, W_slice, bias, tau, lse, ws, stream=None):
    st = _lib.fs_stats(ctypes.byref(shape), _ptr(x_mid), _ptr(W_slice), _ptr(bias), _ptr(tau), _ptr(lse), _ptr(ws),
                       ws.numel(), _stream(stream))
    _check("fs_stats", st)


def fs_slice_fwd_lse(shape, x_mid, fx, W_slice, bias, tau, lse, tokens, wsum, finalize, ws, stream=None):
    st = _lib.fs_slice_fwd_lse(ctypes.byref(shape), _ptr(x_mid), _ptr(fx), _ptr(W_slice), _ptr(bias), _ptr(tau),
                               _ptr(lse), _ptr(tokens), _ptr(wsum), int(bool(finalize)), _ptr(ws), ws.numel(),
                               _stream(stream))
    _check("fs_slice_fwd_lse", st)


def fs_mix_channels(shape, Wc, tokens, tokens_mixed, stream=None):
    _check("fs_mix_channels", _lib.fs_mix_channels(ctypes.byref(shape), _ptr(Wc), _ptr(tokens), _ptr(tokens_mixed),
                                                   _stream(stream)))


def fs_mix_channels_bwd(shape, Wc, tokens, d_tokens_mixed, d_tokens, dWc, stream=None):
    _check("fs_mix_channels_bwd", _lib.fs_mix_channels_bwd(ctypes.byref(shape), _ptr(Wc), _ptr(tokens),
                                                           _ptr(d_tokens_mixed), _ptr(d_tokens), _ptr(dWc),
                                                           _stream(stream)))


def fs_mix_channels_bwd_add(shape, Wc, tokens, d_tokens_mixed, d_tokens, dWc, stream=None):
    _check("fs_mix_channels_bwd_add",
           _lib.fs_mix_channels_bwd_add(ctypes.byref(shape), _ptr(Wc), _ptr(tokens), _ptr(d_tokens_mixed),
                                        _ptr(d_tokens), _ptr(dWc), _stream(stream)))


def fs_slice_finalize(shape, tokens, wsum, stream=None):
    _check("fs_slice_finalize", _lib.fs_slice_finalize(ctypes.byref(shape), _ptr(tokens), _ptr(wsum),
                                                       _stream(stream)))


def fs_mix(shape, M, tokens, tokens_mixed, stream=None):
    _check("fs_mix", _lib.fs_mix(ctypes.byref(shape), _ptr(M), _ptr(tokens), _ptr(tokens_mixed), _stream(stream)))


def fs_deslice_fwd(shape, x_mid, W_slice, bias, tau, tokens_mixed, lse, out, ws, stream=None):
    st = _lib.fs_deslice_fwd(ctypes.byref(shape), _ptr(x_mid), _ptr(W_slice), _ptr(bias), _ptr(tau),
                             _ptr(tokens_mixed), _ptr(lse), _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check("fs_deslice_fwd", st)


def fs_deslice_bwd(shape, x_mid, W_slice, bias, tau, tokens_mixed, lse, dout, d_tokens_mixed, dx_mid, dW, dbias,
                   dtau, accumulate, ws, stream=None):
    st = _lib.fs_deslice_bwd(ctypes.byref(shape), _ptr(x_mid), _ptr(W_slice), _ptr(bias), _ptr(tau),
                             _ptr(tokens_mixed), _ptr(lse), _ptr(dout), _ptr(d_tokens_mixed), _ptr(dx_mid),
                             _ptr(dW), _ptr(dbias), _ptr(dtau), int(bool(accumulate)), _ptr(ws), ws.numel(),
                             _stream(stream))
    _check("fs_deslice_bwd", st)


def fs_mix_bwd(shape, M, tokens, d_tokens_mixed, d_tokens, dM, stream=None):
    st = _lib.fs_mix_bwd(ctypes.byref(shape), _ptr(M), _ptr(tokens), _ptr(d_tokens_mixed), _ptr(d_tokens),
                         _ptr(dM), _stream(stream))
    _check("fs_mix_bwd", st)


def fs_slice_bwd(shape, x_mid, fx, W_slice, bias, tau, tokens, wsum, lse, d_tokens, dx_mid, dfx, dW, dbias, dtau,
                 accumulate, ws, stream=None):
    st = _lib.fs_slice_bwd(ctypes.byref(shape), _ptr(x_mid), _ptr(fx), _ptr(W_slice), _ptr(bias), _ptr(tau),
                           _ptr(tokens), _ptr(wsum), _ptr(lse), _ptr(d_tokens), _ptr(dx_mid), _ptr(dfx), _ptr(dW),
                           _ptr(dbias), _ptr(dtau), int(bool(accumulate)), _ptr(ws), ws.numel(), _stream(stream))
    _check("fs_slice_bwd", st)


def fs_coupling_bwd(shape, x_mid, fx, W_slice, bias, tau, M, tokens, wsum, tokens_mixed, lse, dout, d_tokens_mixed,
                    d_tokens, dx_mid, dfx, dW, dbias, dtau, dM, accumulate, ws, stream=None):
    st = _lib.fs_coupling_bwd(ctypes.byref(shape), _ptr(x_mid), _ptr(fx), _ptr(W_slice), _ptr(bias), _ptr(tau),
                              _ptr(M), _ptr(tokens), _ptr(wsum), _ptr(tokens_mixed), _ptr(lse), _ptr(dout),
                              _ptr(d_tokens_mixed), _ptr(d_tokens), _ptr(dx_mid), _ptr(dfx), _ptr(dW), _ptr(dbias),
                              _ptr(dtau), _ptr(dM), int(bool(accumulate)), _ptr(ws), ws.numel(), _stream(stream))
    _check("fs_coupling_bwd", st)


def fs_device_status(ws, stream=None) -> int:
    return int(_lib.fs_device_status(_ptr(ws), _stream(stream)))


def fs_slice_fwd_noalloc(shape, x_mid, fx, W_slice, bias, tau, tokens, wsum, lse, finalize, stream=None) -> int:
    """fs_slice_fwd on the library's fixed device scratch (no workspace argument, nothing
    allocated).  Returns the scratch's device address, for device_status_at."""
    addr = _P()
    st = _lib.fs_slice_fwd_noalloc(ctypes.byref(shape), _ptr(x_mid), _ptr(fx), _ptr(W_slice), _ptr(bias),
                                   _ptr(tau), _ptr(tokens), _ptr(wsum), _ptr(lse), int(bool(finalize)),
                                   ctypes.byref(addr), _stream(stream))
    _check("fs_slice_fwd_noalloc", st)
    return int(addr.value)


def device_status_at(addr: int, stream=None) -> int:
    """fs_device_status of a scratch given by its device address."""
    return int(_lib.fs_device_status(_P(addr), _stream(stream)))


# ---- argument checks ----------------------------------------------------------------------
#
# The calls below know the size and type of every argument, so they check each tensor here: a
# wrong one raises ValueError before the library sees a pointer.


def _arg(fn, name, t, dtype, numel, dev, optional=False):
    if t is None:
        if optional:
            return None
        raise ValueError(f"{fn}: {name} is missing")
    if t.dtype is dtype and t.numel() == numel and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if t.dtype is not dtype or t.numel() != numel:
        raise ValueError(f"{fn}: {name} has {t.numel()} values of {t.dtype}, expected {numel} of {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{fn}: {name} must be contiguous")
    raise ValueError(f"{fn}: {name} is on {t.device}, the call on the current device and its stream")


# The handle of a device's current stream, without the object around it where torch has that (a
# microsecond of a small call's nine).
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _where(fn, first, stream):
    """The current device, and the raw stream of the call."""
    if not isinstance(first, torch.Tensor) or not first.is_cuda:  # nothing to ask a device for
        return -2, None
    dev = torch.cuda.current_device()
    if stream is None:
        return dev, _current_raw_stream(dev)
    if stream.device_index != dev:
        raise ValueError(f"{fn}: the stream is on cuda:{stream.device_index}, the current device is cuda:{dev}")
    return dev, stream.cuda_stream


# ---- token attention ----------------------------------------------------------------------


def make_attn_shape(B, H, G, d, Hkv=None, Gk=None, scale=None, cap=0.0, prefix=False) -> fs_attn_shape:
    """G query tokens and Gk (default G) key tokens per head; Hkv (default H) key heads; scale
    defaults to 1 / sqrt(d); cap 0 for none; prefix: the prefix mask (FS_MASK_PREFIX)."""
    return fs_attn_shape(int(B), int(H), int(H if Hkv is None else Hkv), int(G), int(G if Gk is None else Gk), int(d),
                         FS_MASK_PREFIX if prefix else FS_MASK_NONE,
                         float(d ** -0.5 if scale is None else scale), float(cap))


class attn_mask:
    """The optional tensors of an attention call: slopes [H], pos_q [B, Gq] and pos_k [B, Gk] (float32);
    doc_q, doc_k, prefix [B] (int32)."""

    def __init__(self, slopes=None, pos_q=None, pos_k=None, doc_q=None, doc_k=None, prefix=None):
        self.slopes, self.pos_q, self.pos_k = slopes, pos_q, pos_k
        self.doc_q, self.doc_k, self.prefix = doc_q, doc_k, prefix


def _attn_mask(fn, s, m, dev):
    """The struct for the tensors that are there, or None (a small call notices each look at one that is not)."""
    if m is None:
        return None
    slopes, pos_q, pos_k, doc_q, doc_k, prefix = m.slopes, m.pos_q, m.pos_k, m.doc_q, m.doc_k, m.prefix
    if slopes is pos_q is pos_k is doc_q is doc_k is prefix is None:
        return None
    c, f, i = fs_attn_mask(), torch.float32, torch.int32
    if slopes is not None:
        c.slopes = _arg(fn, "slopes", slopes, f, s.H, dev)
    if pos_q is not None:
        c.pos_q = _arg(fn, "pos_q", pos_q, f, s.B * s.Gq, dev)
    if pos_k is not None:
        c.pos_k = _arg(fn, "pos_k", pos_k, f, s.B * s.Gk, dev)
    if doc_q is not None:
        c.doc_q = _arg(fn, "doc_q", doc_q, i, s.B * s.Gq, dev)
    if doc_k is not None:
        c.doc_k = _arg(fn, "doc_k", doc_k, i, s.B * s.Gk, dev)
    if prefix is not None:
        c.prefix = _arg(fn, "prefix", prefix, i, s.B, dev)
    return ctypes.byref(c)


def attn_workspace_bytes(shape: fs_attn_shape, backward=False) -> int:
    return int(_lib.fs_attn_workspace_bytes(ctypes.byref(shape), int(bool(backward))))


def attn_path_for_shape(shape: fs_attn_shape, backward=False) -> int:
    """0: warps; 1: tcgen05."""
    return int(_lib.fs_attn_path_for_shape(ctypes.byref(shape), int(bool(backward))))


def attn_workspace(shape: fs_attn_shape, backward=False, device="cuda") -> torch.Tensor:
    """Scratch of fs_attn_fwd, or of fs_attn_bwd."""
    ws = torch.empty(max(16, attn_workspace_bytes(shape, backward)), dtype=torch.uint8, device=device)
    ws[:16].zero_()
    return ws


def fs_attn_fwd(shape, q, k, v, mask, out, lse, ws, stream=None):
    """mask: an attn_mask, or None."""
    fn, s, f = "fs_attn_fwd", shape, torch.float32
    dev, st = _where(fn, q, stream)
    nr, nk = s.B * s.H * s.Gq, s.B * s.Hkv * s.Gk * s.d
    nq, nw = nr * s.d, 0 if ws is None else ws.numel()
    _check(fn, _lib.fs_attn_fwd(
        s, _arg(fn, "q", q, f, nq, dev), _arg(fn, "k", k, f, nk, dev), _arg(fn, "v", v, f, nk, dev),
        _attn_mask(fn, s, mask, dev), _arg(fn, "out", out, f, nq, dev), _arg(fn, "lse", lse, f, nr, dev),
        _arg(fn, "ws", ws, torch.uint8, nw, dev), nw, st))


def fs_attn_bwd(shape, q, k, v, mask, out, lse, dout, dq, dk, dv, ws, stream=None):
    fn, s, f = "fs_attn_bwd", shape, torch.float32
    dev, st = _where(fn, q, stream)
    nr, nk = s.B * s.H * s.Gq, s.B * s.Hkv * s.Gk * s.d
    nq, nw = nr * s.d, 0 if ws is None else ws.numel()
    _check(fn, _lib.fs_attn_bwd(
        s, _arg(fn, "q", q, f, nq, dev), _arg(fn, "k", k, f, nk, dev), _arg(fn, "v", v, f, nk, dev),
        _attn_mask(fn, s, mask, dev), _arg(fn, "out", out, f, nq, dev), _arg(fn, "lse", lse, f, nr, dev),
        _arg(fn, "dout", dout, f, nq, dev), _arg(fn, "dq", dq, f, nq, dev), _arg(fn, "dk", dk, f, nk, dev),
        _arg(fn, "dv", dv, f, nk, dev), _arg(fn, "ws", ws, torch.uint8, nw, dev), nw, st))


# ---- layer norm and 8-bit checkpoints -----------------------------------------------------


def make_rows(rows, C, dtype=FS_F32) -> fs_rows:
    """rows rows of C channels in dtype (a torch.dtype or FS_F32 / FS_BF16)."""
    if isinstance(dtype, torch.dtype):
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"rows are float32 or bfloat16, not {dtype}")
        dtype = FS_BF16 if dtype == torch.bfloat16 else FS_F32
    return fs_rows(int(rows), int(C), int(dtype))


def rows_of(x: torch.Tensor, C=None) -> fs_rows:
    """The rows of x: its last dimension's channels, or C of them (the last dimensions together)."""
    C = x.shape[-1] if C is None else C
    return make_rows(x.numel() // C, C, x.dtype)


def _row_sizes(r):
    dt = torch.bfloat16 if r.dtype == FS_BF16 else torch.float32
    return dt, r.rows * r.C, r.rows * ((r.C + 31) // 32)


def checkpoint(rows: fs_rows, device="cuda"):
    """Buffers (q8, e8) of an 8-bit checkpoint of these rows."""
    return (torch.empty(rows.rows, rows.C, dtype=torch.int8, device=device),
            torch.empty(rows.rows, (rows.C + 31) // 32, dtype=torch.uint8, device=device))


def norm_workspace_bytes(rows: fs_rows) -> int:
    return int(_lib.fs_norm_workspace_bytes(ctypes.byref(rows)))


def norm_workspace(rows: fs_rows, device="cuda") -> torch.Tensor:
    """Scratch for fs_norm_bwd."""
    ws = torch.empty(max(16, norm_workspace_bytes(rows)), dtype=torch.uint8, device=device)
    ws[:16].zero_()
    return ws


def fs_norm_fwd(rows, x, res, gamma, beta, eps, sum, y, mean, rstd, q8=None, e8=None, stream=None):
    fn, f, r, C = "fs_norm_fwd", torch.float32, rows.rows, rows.C
    dt, n, nb = _row_sizes(rows)
    dev, st = _where(fn, x, stream)
    _check(fn, _lib.fs_norm_fwd(
        rows, _arg(fn, "x", x, dt, n, dev), _arg(fn, "res", res, dt, n, dev, True),
        _arg(fn, "gamma", gamma, f, C, dev, True), _arg(fn, "beta", beta, f, C, dev, True), eps,
        _arg(fn, "sum", sum, dt, n, dev, True), _arg(fn, "y", y, dt, n, dev), _arg(fn, "mean", mean, f, r, dev, True),
        _arg(fn, "rstd", rstd, f, r, dev, True), _arg(fn, "q8", q8, torch.int8, n, dev, True),
        _arg(fn, "e8", e8, torch.uint8, nb, dev, True), st))


def fs_norm_bwd(rows, v, q8, e8, gamma, mean, rstd, dy, dres, dv, dgamma, dbeta, accumulate, ws, stream=None):
    fn, f, r, C = "fs_norm_bwd", torch.float32, rows.rows, rows.C
    dt, n, nb = _row_sizes(rows)
    dev, st = _where(fn, dy, stream)
    nw = 0 if ws is None else ws.numel()
    _check(fn, _lib.fs_norm_bwd(
        rows, _arg(fn, "v", v, dt, n, dev, True), _arg(fn, "q8", q8, torch.int8, n, dev, True),
        _arg(fn, "e8", e8, torch.uint8, nb, dev, True), _arg(fn, "gamma", gamma, f, C, dev, True),
        _arg(fn, "mean", mean, f, r, dev), _arg(fn, "rstd", rstd, f, r, dev), _arg(fn, "dy", dy, dt, n, dev),
        _arg(fn, "dres", dres, dt, n, dev, True), _arg(fn, "dv", dv, dt, n, dev),
        _arg(fn, "dgamma", dgamma, f, C, dev, True), _arg(fn, "dbeta", dbeta, f, C, dev, True), int(bool(accumulate)),
        _arg(fn, "ws", ws, torch.uint8, nw, dev), nw, st))


def fs_ckpt_pack(rows, x, q8, e8, stream=None):
    fn = "fs_ckpt_pack"
    dt, n, nb = _row_sizes(rows)
    dev, st = _where(fn, x, stream)
    _check(fn, _lib.fs_ckpt_pack(rows, _arg(fn, "x", x, dt, n, dev), _arg(fn, "q8", q8, torch.int8, n, dev),
                                 _arg(fn, "e8", e8, torch.uint8, nb, dev), st))


def fs_ckpt_unpack(rows, q8, e8, x, stream=None):
    fn = "fs_ckpt_unpack"
    dt, n, nb = _row_sizes(rows)
    dev, st = _where(fn, x, stream)
    _check(fn, _lib.fs_ckpt_unpack(rows, _arg(fn, "q8", q8, torch.int8, n, dev),
                                   _arg(fn, "e8", e8, torch.uint8, nb, dev), _arg(fn, "x", x, dt, n, dev), st))


# ---- linear maps and dropout ---------------------------------------------------------------


def make_linear(rows, Cin, Cout, dtype=FS_F32) -> fs_linear:
    """rows rows of Cin channels to rows of Cout, in dtype (a torch.dtype or FS_F32 / FS_BF16)."""
    r = make_rows(rows, Cin, dtype)
    return fs_linear(r.rows, r.C, int(Cout), r.dtype)


def linear_workspace_bytes(s: fs_linear, backward=False) -> int:
    return int(_lib.fs_linear_workspace_bytes(ctypes.byref(s), int(bool(backward))))


def linear_path_for_shape(s: fs_linear, backward=False) -> int:
    """0: fp32 multiply-adds; 1: tcgen05."""
    return int(_lib.fs_linear_path_for_shape(ctypes.byref(s), int(bool(backward))))


def linear_workspace(s: fs_linear, backward=False, device="cuda") -> torch.Tensor:
    """Scratch of fs_linear_fwd, or of fs_linear_bwd."""
    ws = torch.empty(max(16, linear_workspace_bytes(s, backward)), dtype=torch.uint8, device=device)
    ws[:16].zero_()
    return ws


def dropout_rng(seed, offset=0, device="cuda") -> torch.Tensor:
    """The two words {seed, offset} of a dropout (taken modulo 2^64), which `rng` arguments want."""
    return torch.tensor([((int(w) + (1 << 63)) % (1 << 64)) - (1 << 63) for w in (seed, offset)], dtype=torch.int64,
                        device=device)


def fs_linear_fwd(s, x, W, bias, act, p, rng, res, y, pre, ws, stream=None):
    """act: FS_ACT_*; rng: see dropout_rng, None without dropout; bias, res, pre may be None."""
    fn, ci, co, r = "fs_linear_fwd", s.Cin, s.Cout, s.rows
    dt, ny = torch.bfloat16 if s.dtype == FS_BF16 else torch.float32, r * co
    dev, st = _where(fn, x, stream)
    nw = 0 if ws is None else ws.numel()
    _check(fn, _lib.fs_linear_fwd(
        s, _arg(fn, "x", x, dt, r * ci, dev), _arg(fn, "W", W, dt, co * ci, dev),
        _arg(fn, "bias", bias, torch.float32, co, dev, True), act, p, _arg(fn, "rng", rng, torch.int64, 2, dev, True),
        _arg(fn, "res", res, dt, ny, dev, True), _arg(fn, "y", y, dt, ny, dev), _arg(fn, "pre", pre, dt, ny, dev, True),
        _arg(fn, "ws", ws, torch.uint8, nw, dev), nw, st))


def fs_linear_bwd(s, x, W, g, act, p, rng, pre, dres, dx, dW, dbias, accumulate, ws, stream=None):
    """act, p, rng, pre: of the call that made x; x, W, pre, dres, dx, dW, dbias may be None (see the header)."""
    fn, ci, co, r, f = "fs_linear_bwd", s.Cin, s.Cout, s.rows, torch.float32
    dt, nx = torch.bfloat16 if s.dtype == FS_BF16 else torch.float32, r * ci
    dev, st = _where(fn, g, stream)
    nw = 0 if ws is None else ws.numel()
    _check(fn, _lib.fs_linear_bwd(
        s, _arg(fn, "x", x, dt, nx, dev, True), _arg(fn, "W", W, dt, co * ci, dev, True),
        _arg(fn, "g", g, dt, r * co, dev), act, p, _arg(fn, "rng", rng, torch.int64, 2, dev, True),
        _arg(fn, "pre", pre, dt, nx, dev, True), _arg(fn, "dres", dres, dt, nx, dev, True),
        _arg(fn, "dx", dx, dt, nx, dev, True), _arg(fn, "dW", dW, f, co * ci, dev, True),
        _arg(fn, "dbias", dbias, f, co, dev, True), int(bool(accumulate)), _arg(fn, "ws", ws, torch.uint8, nw, dev), nw,
        st))


def fs_dropout_fwd(rows, x, act, p, rng, res, y, stream=None):
    """act: FS_ACT_*; rng: see dropout_rng, None for p = 0; res may be None."""
    fn = "fs_dropout_fwd"
    dt, n, _ = _row_sizes(rows)
    dev, st = _where(fn, x, stream)
    _check(fn, _lib.fs_dropout_fwd(
        rows, _arg(fn, "x", x, dt, n, dev), act, p, _arg(fn, "rng", rng, torch.int64, 2, dev, True),
        _arg(fn, "res", res, dt, n, dev, True), _arg(fn, "y", y, dt, n, dev), st))


def fs_dropout_bwd(rows, dy, act, p, rng, pre, dx, stream=None):
    fn = "fs_dropout_bwd"
    dt, n, _ = _row_sizes(rows)
    dev, st = _where(fn, dy, stream)
    _check(fn, _lib.fs_dropout_bwd(
        rows, _arg(fn, "dy", dy, dt, n, dev), act, p, _arg(fn, "rng", rng, torch.int64, 2, dev, True),
        _arg(fn, "pre", pre, dt, n, dev, True), _arg(fn, "dx", dx, dt, n, dev), st))


# ---- convenience: one coupling, buffers allocated through torch ----------------------------


class Coupling:
    """Allocates the outputs and scratch of one slice -> mix -> deslice coupling
    (forward, and backward when asked) once, then runs it through the C ABI."""

    def __init__(self, B, N, H, d, G, dtype=torch.bfloat16, eps=1e-5, backward=False, device="cuda", dot=None):
        # A coupling that will be differentiated defaults to the split products
        # (FS_DOT_BF16X2): the temperature gradient is a near-cancelling sum that
        # bf16 tokens cannot resolve.
        if dot is None:
            dot = FS_DOT_BF16X2 if backward else FS_DOT_BF16
        self.shape = make_shape(B, N, H, d, G, dtype, eps, dot)
        self.dtype = dtype
        f32 = dict(dtype=torch.float32, device=device)
        self.tokens = torch.empty(B, H, G, d, **f32)
        self.wsum = torch.empty(B, H, G, **f32)
        self.lse = torch.empty(B, H, N, **f32)
        self.tokens_mixed = torch.empty(B, H, G, d, **f32)
        self.out = torch.empty(B, N, H, d, dtype=dtype, device=device)
        self.ws_slice = workspace(self.shape, FS_OP_SLICE_FWD, device)
        self.ws_deslice = workspace(self.shape, FS_OP_DESLICE_FWD, device)
        if backward:
            self.d_tokens_mixed = torch.empty(B, H, G, d, **f32)
            self.d_tokens = torch.empty(B, H, G, d, **f32)
            self.dx_mid = torch.empty(B, N, H, d, dtype=dtype, device=device)
            self.dfx = torch.empty(B, N, H, d, dtype=dtype, device=device)
            self.dW = torch.empty(H, d, G, **f32)
            self.dbias = torch.empty(H, G, **f32)
            self.dtau = torch.empty(H, **f32)
            self.dM = torch.empty(H, G, G, **f32)
            self.ws_dbwd = workspace(self.shape, FS_OP_DESLICE_BWD, device)
            self.ws_sbwd = workspace(self.shape, FS_OP_SLICE_BWD, device)
            self.ws_cbwd = workspace(self.shape, FS_OP_COUPLING_BWD, device)

    def forward(self, x_mid, fx, W_slice, bias, tau, M, stream=None):
        s = self.shape
        fs_slice_fwd(s, x_mid, fx, W_slice, bias, tau, self.tokens, self.wsum, self.lse, True, self.ws_slice, stream)
        fs_mix(s, M, self.tokens, self.tokens_mixed, stream)
        fs_deslice_fwd(s, x_mid, W_slice, bias, tau, self.tokens_mixed, self.lse, self.out, self.ws_deslice, stream)
        return self.out

    def backward(self, x_mid, fx, W_slice, bias, tau, M, dout, stream=None, fused=True):
        """fused: one fs_coupling_bwd call; else fs_deslice_bwd, fs_mix_bwd, fs_slice_bwd."""
        s = self.shape
        if fused:
            fs_coupling_bwd(s, x_mid, fx, W_slice, bias, tau, M, self.tokens, self.wsum, self.tokens_mixed, self.lse,
                            dout, self.d_tokens_mixed, self.d_tokens, self.dx_mid, self.dfx, self.dW, self.dbias,
                            self.dtau, self.dM, False, self.ws_cbwd, stream)
        else:
            fs_deslice_bwd(s, x_mid, W_slice, bias, tau, self.tokens_mixed, self.lse, dout, self.d_tokens_mixed,
                           self.dx_mid, self.dW, self.dbias, self.dtau, False, self.ws_dbwd, stream)
            fs_mix_bwd(s, M, self.tokens, self.d_tokens_mixed, self.d_tokens, self.dM, stream)
            fs_slice_bwd(s, x_mid, fx, W_slice, bias, tau, self.tokens, self.wsum, self.lse, self.d_tokens,
                         self.dx_mid, self.dfx, self.dW, self.dbias, self.dtau, True, self.ws_sbwd, stream)
        return {"dx_mid": self.dx_mid, "dfx": self.dfx, "dW": self.dW, "dbias": self.dbias, "dtau": self.dtau,
                "dM": self.dM}

    def device_status(self, stream=None):
        worst = FS_OK
        for ws in (self.ws_slice, self.ws_deslice) + (
                (self.ws_dbwd, self.ws_sbwd, self.ws_cbwd) if hasattr(self, "ws_dbwd") else ()):
            st = fs_device_status(ws, stream)
            worst = worst or st
        return worst


class AttentionCoupling:
    """A coupling with the original layer's token operation, self-attention of a head's G tokens:

      tokens = slice(x_mid, fx);  q, k, v = Wq, Wk, Wv tokens (per head, [H, d, d]);
      tokens_mixed = attention(q, k, v);  out = deslice(x_mid, tokens_mixed)

    cap, prefix, and the mask of the calls: see make_attn_shape and attn_mask.
    qk_norm: q and k pass through a layer norm over their d channels, with weights gamma_q, gamma_k
    [d] (None: 1); it bounds the scores whatever the tokens' size.
    checkpointed: nothing but the 8-bit checkpoints of x_mid and fx is kept for the backward pass,
    which restores them into `restored` (a pair of buffers [B, N, H, d], which layers may share:
    pass another layer's) and computes the tokens again.  Its gradients are those at the restored
    inputs.  The buffers that the forward fills are scratch then, too."""

    NORM_EPS = 1e-5

    def __init__(self, B, N, H, d, G, dtype=torch.bfloat16, eps=1e-5, backward=False, device="cuda", dot=None,
                 cap=0.0, prefix=False, qk_norm=False, checkpointed=False, restored=None):
        if checkpointed and not backward:
            raise ValueError("a checkpoint is for the backward pass")
        if dot is None:
            dot = FS_DOT_BF16X2 if backward else FS_DOT_BF16
        self.shape = make_shape(B, N, H, d, G, dtype, eps, dot)
        self.attn = make_attn_shape(B, H, G, d, cap=cap, prefix=prefix)
        self.token_rows = make_rows(B * H * G, d)
        self.qk_norm, self.checkpointed = qk_norm, checkpointed
        f32 = dict(dtype=torch.float32, device=device)

        def tokens():
            return torch.empty(B, H, G, d, **f32)

        def points():
            return torch.empty(B, N, H, d, dtype=dtype, device=device)

        self.tokens, self.tokens_mixed = tokens(), tokens()
        self.wsum, self.attn_lse = torch.empty(B, H, G, **f32), torch.empty(B, H, G, **f32)
        self.lse = torch.empty(B, H, N, **f32)
        self.q, self.k, self.v = tokens(), tokens(), tokens()
        # what the attention reads, and the norms' statistics
        self.q_in, self.k_in = (tokens(), tokens()) if qk_norm else (self.q, self.k)
        self.stats = [torch.empty(B * H * G, **f32) for _ in range(4)] if qk_norm else [None] * 4
        self.out = points()
        self.ws_slice = workspace(self.shape, FS_OP_SLICE_FWD, device)
        self.ws_deslice = workspace(self.shape, FS_OP_DESLICE_FWD, device)
        self.ws_attn = attn_workspace(self.attn, False, device)
        self.packed = None
        if checkpointed:
            self.point_rows = make_rows(B * N, H * d, dtype)
            self.packed = (checkpoint(self.point_rows, device), checkpoint(self.point_rows, device))
            self.restored = (points(), points()) if restored is None else restored
        if backward:
            self.d_tokens_mixed, self.d_tokens = tokens(), tokens()
            self.dq, self.dk, self.dv = tokens(), tokens(), tokens()
            self.dx_mid, self.dfx = points(), points()
            self.dW = torch.empty(H, d, G, **f32)
            self.dbias, self.dtau = torch.empty(H, G, **f32), torch.empty(H, **f32)
            self.dWq, self.dWk, self.dWv = (torch.empty(H, d, d, **f32) for _ in range(3))
            self.dgamma_q, self.dgamma_k, self.unused = (torch.empty(d, **f32) for _ in range(3))
            self.ws_dbwd = workspace(self.shape, FS_OP_DESLICE_BWD, device)
            self.ws_sbwd = workspace(self.shape, FS_OP_SLICE_BWD, device)
            self.ws_abwd = attn_workspace(self.attn, True, device)
            self.ws_norm = norm_workspace(self.token_rows, device)

    def _mix(self, x_mid, fx, W_slice, bias, tau, Wq, Wk, Wv, mask, gamma_q, gamma_k, stream):
        s, r = self.shape, self.token_rows
        fs_slice_fwd(s, x_mid, fx, W_slice, bias, tau, self.tokens, self.wsum, self.lse, True, self.ws_slice, stream)
        for W, t in ((Wq, self.q), (Wk, self.k), (Wv, self.v)):
            fs_mix_channels(s, W, self.tokens, t, stream)
        if self.qk_norm:
            mq, rq, mk, rk = self.stats
            fs_norm_fwd(r, self.q, None, gamma_q, None, self.NORM_EPS, None, self.q_in, mq, rq, stream=stream)
            fs_norm_fwd(r, self.k, None, gamma_k, None, self.NORM_EPS, None, self.k_in, mk, rk, stream=stream)
        fs_attn_fwd(self.attn, self.q_in, self.k_in, self.v, mask, self.tokens_mixed, self.attn_lse, self.ws_attn, stream)

    def forward(self, x_mid, fx, W_slice, bias, tau, Wq, Wk, Wv, mask=None, gamma_q=None, gamma_k=None, stream=None):
        self._mix(x_mid, fx, W_slice, bias, tau, Wq, Wk, Wv, mask, gamma_q, gamma_k, stream)
        fs_deslice_fwd(self.shape, x_mid, W_slice, bias, tau, self.tokens_mixed, self.lse, self.out, self.ws_deslice,
                       stream)
        if self.checkpointed:
            for x, (q8, e8) in zip((x_mid, fx), self.packed):
                fs_ckpt_pack(self.point_rows, x, q8, e8, stream)
        return self.out

    def backward(self, x_mid, fx, W_slice, bias, tau, Wq, Wk, Wv, dout, mask=None, gamma_q=None, gamma_k=None,
                 stream=None):
        """x_mid, fx: the forward's, or None from the checkpoint."""
        s, r = self.shape, self.token_rows
        if self.checkpointed:
            if x_mid is not None or fx is not None:
                raise ValueError("x_mid and fx come from the checkpoint")
            for x, (q8, e8) in zip(self.restored, self.packed):
                fs_ckpt_unpack(self.point_rows, q8, e8, x, stream)
            x_mid, fx = self.restored
            self._mix(x_mid, fx, W_slice, bias, tau, Wq, Wk, Wv, mask, gamma_q, gamma_k, stream)
        fs_deslice_bwd(s, x_mid, W_slice, bias, tau, self.tokens_mixed, self.lse, dout, self.d_tokens_mixed,
                       self.dx_mid, self.dW, self.dbias, self.dtau, False, self.ws_dbwd, stream)
        fs_attn_bwd(self.attn, self.q_in, self.k_in, self.v, mask, self.tokens_mixed, self.attn_lse,
                    self.d_tokens_mixed, self.dq, self.dk, self.dv, self.ws_abwd, stream)
        if self.qk_norm:
            for t, g, d, dg, mean, rstd in ((self.q, gamma_q, self.dq, self.dgamma_q, *self.stats[:2]),
                                            (self.k, gamma_k, self.dk, self.dgamma_k, *self.stats[2:])):
                fs_norm_bwd(r, t, None, None, g, mean, rstd, d, None, d, dg, self.unused, False, self.ws_norm, stream)
        fs_mix_channels_bwd(s, Wq, self.tokens, self.dq, self.d_tokens, self.dWq, stream)
        fs_mix_channels_bwd_add(s, Wk, self.tokens, self.dk, self.d_tokens, self.dWk, stream)
        fs_mix_channels_bwd_add(s, Wv, self.tokens, self.dv, self.d_tokens, self.dWv, stream)
        fs_slice_bwd(s, x_mid, fx, W_slice, bias, tau, self.tokens, self.wsum, self.lse, self.d_tokens, self.dx_mid,
                     self.dfx, self.dW, self.dbias, self.dtau, True, self.ws_sbwd, stream)
        g = {"dx_mid": self.dx_mid, "dfx": self.dfx, "dW": self.dW, "dbias": self.dbias, "dtau": self.dtau,
             "dWq": self.dWq, "dWk": self.dWk, "dWv": self.dWv}
        if self.qk_norm:
            g.update(dgamma_q=self.dgamma_q, dgamma_k=self.dgamma_k)
        return g

    def device_status(self, stream=None):
        worst = FS_OK
        for ws in (self.ws_slice, self.ws_deslice, self.ws_attn) + (
                (self.ws_dbwd, self.ws_sbwd, self.ws_abwd, self.ws_norm) if hasattr(self, "ws_dbwd") else ()):
            st = fs_device_status(ws, stream)
            worst = worst or st
        return worst


class ShardedCoupling:
    """The local compute of a point-sharded coupling (App. G.4) for
    sharding.sharded_forward / sharding.sharded_backward: this rank's points of
    every batch, x_mid and fx [B, n_local, H, d], through the C ABI.  The slice
    keeps its numerators unnormalised (finalize = 0) until they are summed over
    ranks; the backward's two calls add into the same dx_mid, dW, dbias, dtau."""

    def __init__(self, B, n_local, H, d, G, x_mid, fx, W_slice, bias, tau, M, dtype=torch.bfloat16, eps=1e-5,
                 dout=None, device="cuda", dot=None):
        self.c = Coupling(B, n_local, H, d, G, dtype, eps, backward=dout is not None, device=device, dot=dot)
        self.x, self.fx, self.W, self.bias, self.tau, self.M, self.dout = x_mid, fx, W_slice, bias, tau, M, dout

    def slice_partials(self):
        c = self.c
        fs_slice_fwd(c.shape, self.x, self.fx, self.W, self.bias, self.tau, c.tokens, c.wsum, c.lse, False,
                     c.ws_slice)
        return c.tokens, c.wsum

    def finalize(self, U, S):
        fs_slice_finalize(self.c.shape, U, S)
        return U

    def mix(self, tokens):
        fs_mix(self.c.shape, self.M, tokens, self.c.tokens_mixed)
        return self.c.tokens_mixed

    def deslice(self, tokens_mixed):
        c = self.c
        fs_deslice_fwd(c.shape, self.x, self.W, self.bias, self.tau, tokens_mixed, c.lse, c.out, c.ws_deslice)
        return c.out

    def deslice_bwd(self):
        c = self.c
        fs_deslice_bwd(c.shape, self.x, self.W, self.bias, self.tau, c.tokens_mixed, c.lse, self.dout,
                       c.d_tokens_mixed, c.dx_mid, c.dW, c.dbias, c.dtau, False, c.ws_dbwd)
        return c.d_tokens_mixed

    def mix_bwd(self, d_tokens_mixed):
        c = self.c
        fs_mix_bwd(c.shape, self.M, c.tokens, d_tokens_mixed, c.d_tokens, c.dM)
        return c.d_tokens, c.dM

    def slice_bwd(self, d_tokens):
        c = self.c
        fs_slice_bwd(c.shape, self.x, self.fx, self.W, self.bias, self.tau, c.tokens, c.wsum, c.lse, d_tokens,
                     c.dx_mid, c.dfx, c.dW, c.dbias, c.dtau, True, c.ws_sbwd)
        return c.dW, c.dbias, c.dtau


class FeedForward:
    """The second half of a layer, behind its norm: y = res + drop(W2 drop(act(W1 x + b1)) + b2), on rows of C
    channels with `hidden` between, with its buffers allocated once.

    p: both dropouts' rate; rng_hidden, rng_out: their words (dropout_rng), which differ from each other and
    from other layers' and steps', and which the backward gets again.  backward: the buffers of the gradients,
    too; the forward then keeps x (a reference), the pre-activations and the hidden rows."""

    def __init__(self, rows, C, hidden, dtype=torch.bfloat16, act=FS_ACT_GELU, p=0.0, backward=False, device="cuda"):
        self.first, self.second = make_linear(rows, C, hidden, dtype), make_linear(rows, hidden, C, dtype)
        self.rows, self.act, self.p = make_rows(rows, C, dtype), act, p
        own = dict(dtype=dtype, device=device)
        self.h, self.y = torch.empty(rows, hidden, **own), torch.empty(rows, C, **own)
        self.pre, self.x = (torch.empty(rows, hidden, **own) if backward else None), None
        self.ws = [linear_workspace(s, False, device) for s in (self.first, self.second)]
        if backward:
            f32 = dict(dtype=torch.float32, device=device)
            self.g, self.dh, self.dx = torch.empty(rows, C, **own), torch.empty(rows, hidden, **own), torch.empty(rows, C, **own)
            self.dW1, self.db1 = torch.empty(hidden, C, **f32), torch.empty(hidden, **f32)
            self.dW2, self.db2 = torch.empty(C, hidden, **f32), torch.empty(C, **f32)
            self.ws_bwd = [linear_workspace(s, True, device) for s in (self.first, self.second)]

    def forward(self, x, W1, b1, W2, b2, res=None, rng_hidden=None, rng_out=None, stream=None):
        self.x = x
        fs_linear_fwd(self.first, x, W1, b1, self.act, self.p, rng_hidden, None, self.h, self.pre, self.ws[0], stream)
        fs_linear_fwd(self.second, self.h, W2, b2, FS_ACT_NONE, self.p, rng_out, res, self.y, None, self.ws[1], stream)
        return self.y

    def backward(self, W1, W2, dy, dres=None, rng_hidden=None, rng_out=None, accumulate=False, stream=None):
        """dy: the gradient of y (the residual's own gradient, too); dres: added to that of x."""
        g = dy
        if self.p > 0:
            fs_dropout_bwd(self.rows, dy, FS_ACT_NONE, self.p, rng_out, None, self.g, stream)
            g = self.g
        fs_linear_bwd(self.second, self.h, W2, g, self.act, self.p, rng_hidden, self.pre, None, self.dh, self.dW2, self.db2,
                      accumulate, self.ws_bwd[1], stream)
        fs_linear_bwd(self.first, self.x, W1, self.dh, FS_ACT_NONE, 0.0, None, None, dres, self.dx, self.dW1, self.db1,
                      accumulate, self.ws_bwd[0], stream)
        return {"dx": self.dx, "dW1": self.dW1, "db1": self.db1, "dW2": self.dW2, "db2": self.db2}
