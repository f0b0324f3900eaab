"""fp64 oracle of the operators around the coupling (numpy, materialised): layer norm, the
8-bit checkpoint, and the attention of the slice tokens.  Test infrastructure only; it shares
no code with the library."""
from __future__ import annotations

import numpy as np

from . import flashslice_oracle as fso

BLOCK = 32


def norm(v, gamma=None, beta=None, eps=1e-5):
    """y, mean, rstd of the rows of v [R, C]."""
    v = np.asarray(v, np.float64)
    mean = v.mean(1)
    rstd = 1.0 / np.sqrt(((v - mean[:, None]) ** 2).mean(1) + eps)
    y = (v - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean, rstd


def norm_bwd(v, gamma, mean, rstd, dy, dres=None):
    """dv, dgamma, dbeta with the given statistics (those of v for the gradient of norm)."""
    v, dy = np.asarray(v, np.float64), np.asarray(dy, np.float64)
    mean, rstd = np.asarray(mean, np.float64)[:, None], np.asarray(rstd, np.float64)[:, None]
    xh = (v - mean) * rstd
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dv = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    if dres is not None:
        dv = dv + np.asarray(dres, np.float64)
    return dv, (dy * xh).sum(0), dy.sum(0)


def pack(x):
    """q [R, C] and the scale exponents' bytes [R, ceil(C / 32)] of x, block by block."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    q, e = np.zeros((R, C), np.int8), np.zeros((R, -(-C // BLOCK)), np.uint8)
    for r in range(R):
        for b in range(e.shape[1]):
            f = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(f).all():
                e[r, b] = 255
                continue
            s = -126  # the smallest exponent at which every rounded magnitude is at most 127
            if np.abs(f).max() > 0:
                s = max(s, int(np.frexp(np.abs(f).max())[1]) - 8)
            while np.abs(np.rint(np.ldexp(f, -s))).max() > 127:
                s += 1
            q[r, b * BLOCK:(b + 1) * BLOCK] = np.rint(np.ldexp(f, -s))
            e[r, b] = s + 127
    return q, e


def unpack(q, e):
    e = np.repeat(e.astype(np.int64), BLOCK, axis=1)[:, :q.shape[1]]
    return np.where(e == 255, np.nan, np.ldexp(q.astype(np.float64), np.minimum(e, 254) - 127))


def visible(Gq, Gk, doc_q=None, doc_k=None, prefix=None):
    """[Gq, Gk] of one sample: which keys a query sees.  prefix: None for no prefix mask."""
    ok = np.ones((Gq, Gk), bool)
    if doc_q is not None:
        ok &= (doc_q[:, None] == doc_k[None, :]) & (doc_k >= 0)[None, :]
    if prefix is not None:
        i, j = np.arange(Gq)[:, None] + (Gk - Gq), np.arange(Gk)[None, :]
        ok &= (j <= i) | (j < prefix)
    return ok


def attention(q, k, v, scale, cap=0.0, slopes=None, pos_q=None, pos_k=None, doc_q=None, doc_k=None, prefix=None,
              dout=None):
    """out [B, H, Gq, d] and lse [B, H, Gq]; with dout also dq, dk, dv.  Sums run over the visible
    keys alone, so nothing that a mask hides reaches a result."""
    B, H, Gq, d = q.shape
    Hkv, Gk = k.shape[1], k.shape[2]
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    out, lse = np.zeros((B, H, Gq, d)), np.full((B, H, Gq), -np.inf)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        ok = visible(Gq, Gk, None if doc_q is None else doc_q[b], None if doc_k is None else doc_k[b],
                     None if prefix is None else prefix[b])
        for h in range(H):
            g = h // (H // Hkv)
            for i in range(Gq):
                at = np.nonzero(ok[i])[0]
                if not len(at):
                    continue
                kk, vv = k[b, g, at], v[b, g, at]
                s = scale * (kk @ q[b, h, i])
                a = cap * np.tanh(s / cap) if cap else s.copy()
                if slopes is not None:
                    pq = float(i + Gk - Gq) if pos_q is None else float(pos_q[b, i])
                    pk = at.astype(np.float64) if pos_k is None else pos_k[b, at].astype(np.float64)
                    a = a - float(slopes[h]) * np.abs(pq - pk)
                top = a.max()
                if top == -np.inf:  # no key has any weight
                    continue
                p = np.exp(a - top) if np.isfinite(top) else np.full(len(at), np.nan)
                lse[b, h, i] = top + np.log(p.sum())
                p = p / p.sum()
                out[b, h, i] = p @ vv
                if dout is None:
                    continue
                do = np.asarray(dout[b, h, i], np.float64)
                dv[b, g, at] += p[:, None] * do
                ds = p * (vv @ do - out[b, h, i] @ do)
                if cap:
                    ds = ds * (1.0 - np.tanh(s / cap) ** 2)
                ds = ds * scale
                dq[b, h, i] = ds @ kk
                dk[b, g, at] += ds[:, None] * q[b, h, i]
    return (out, lse) if dout is None else (out, lse, dq, dk, dv)


def attention_coupling(x_mid, fx, W_slice, bias, tau, Wq, Wk, Wv, scale, cap=0.0, gamma_q=None, gamma_k=None,
                       qk_norm=False, norm_eps=1e-5, eps=1e-5, dout=None, **mask):
    """slice -> q, k, v maps -> (norms of q and k) -> attention -> deslice; with dout the gradients."""
    s = fso.slice_fwd(x_mid, fx, W_slice, bias, tau, eps)
    z = s["tokens"]
    q, k, v = (fso.mix_channels(W, z) for W in (Wq, Wk, Wv))
    d = q.shape[-1]
    qn, kn, stats = q, k, None
    if qk_norm:
        (yq, mq, rq), (yk, mk, rk) = (norm(t.reshape(-1, d), g, None, norm_eps) for t, g in ((q, gamma_q), (k, gamma_k)))
        qn, kn, stats = yq.reshape(q.shape), yk.reshape(k.shape), (mq, rq, mk, rk)
    tm, lse = attention(qn, kn, v, scale, cap, **mask)
    res = {"out": fso.deslice_fwd(x_mid, W_slice, bias, tau, tm), "tokens": z, "tokens_mixed": tm}
    if dout is None:
        return res
    dd = fso.deslice_bwd(x_mid, W_slice, bias, tau, tm, dout)
    _, _, dq, dk, dv = attention(qn, kn, v, scale, cap, dout=dd["d_tokens_mixed"], **mask)
    if qk_norm:
        shape = q.shape
        dq, dgq, _ = norm_bwd(q.reshape(-1, d), gamma_q, stats[0], stats[1], dq.reshape(-1, d))
        dk, dgk, _ = norm_bwd(k.reshape(-1, d), gamma_k, stats[2], stats[3], dk.reshape(-1, d))
        dq, dk = dq.reshape(shape), dk.reshape(shape)
        res.update(dgamma_q=dgq, dgamma_k=dgk)
    dz = 0.0
    for name, W, g in (("dWq", Wq, dq), ("dWk", Wk, dk), ("dWv", Wv, dv)):
        r = fso.mix_channels_bwd(W, z, g)
        dz = dz + r["d_tokens"]
        res[name] = r["dWc"]
    sb = fso.slice_bwd(x_mid, fx, W_slice, bias, tau, z, s["wsum"], dz, eps)
    res.update({n: dd[n] + sb[n] for n in ("dx_mid", "dW", "dbias", "dtau")}, dfx=sb["dfx"])
    return res
