"""Inputs, calls and error bounds of the linear maps' tests.

Bounds, elementwise, with u = 2^-24 (fp32's half step) and h the rows' half step (bf16 2^-8, fp32
2^-24), of a sum of K products whose magnitudes add up to S:

* fp32 multiply-adds run over at most 128 terms, these sums over K / 128 in each part, and at most
  304 parts, eight at a time (38) and these eight in turn, are added: (128 + K / 128 + 46) u S.
* Tensor cores add 16 products a step and cut their accumulator towards zero, 2 u of it each time.
  Sums with fp32 results are taken out after at most 1024 terms (64 steps, 128 u) and added in fp32, K / 256
  times over all parts at most, in as many chains as there are parts; fp32 operands come in three bf16 parts, which leave out at most 5 u of a
  product.  bf16 results are rounded to 2^-9, and their sums run through: K / 16 steps, K / 8 u.
So fp32 results are within (180 + K / 128) u S and bf16 rows before their rounding (180 + K / 8) u S.

Past the sum a value goes through the activation, whose slope is at most 1.13, and 1 / (1 - p).  The
activation itself is off by at most 8 u of the larger of itself and its argument in fp32 (what a GELU or SILU
takes from its argument is at most half of it, and good to 16 u), 2^-12 of itself and 2e-7 in bf16, where a
slope is off by at most 1.2e-4; in fp32 by 32 u (1 - sigmoid is off by u, times an argument below 17
where it is not exactly 0).  The residual's addition rounds once more."""
import numpy as np
import torch

from oracle import operators_oracle as orc

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
ACTS = ("none", "relu", "gelu", "silu")
SEED, STEP = (1 << 40) + 12345, (7 << 33) + 3


def tensor(rng, shape, dtype, scale=1.0, shift=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale + shift).astype(np.float32)).to("cuda", DTYPES[dtype])


def host(t):
    return None if t is None else t.double().cpu().numpy()


def spare(shape, dtype, extra=64):
    """An output inside a longer buffer: nothing behind it may be written."""
    n = int(np.prod(shape))
    buf = torch.full((n + extra,), 7.0, dtype=dtype, device="cuda")
    return buf[:n].view(shape), buf[n:]


def untouched(*tails):
    return all(bool((t == 7).all()) for t in tails)


def sum_bound(K, S, dtype):
    return (180 + K / (128 if dtype == "f32" else 8)) * U * S


def act_off(a, u, dtype):
    """What the activation's value is off by."""
    if dtype == "f32":
        return 8 * U * np.maximum(np.abs(a), np.abs(u))
    return 2.0 ** -12 * np.abs(a) + 2e-7


def forward_bound(x, W, bias, act, p, res, y, u, dtype):
    S = np.abs(x) @ np.abs(W).T + (0 if bias is None else np.abs(bias))
    du = sum_bound(x.shape[1], S, dtype) + 2 * U * np.abs(u)
    a = orc.activation(act, u)[0]
    da = 1.13 * du + (act_off(a, u, dtype) if act in ("gelu", "silu") else 0)
    dy = (da + 2 * U * np.abs(a)) / (1 - p)
    if res is not None:
        dy = dy + 2 * U * (np.abs(y) + np.abs(res))
    return dy + HALF[dtype] * 1.01 * np.abs(y) + 1e-30, du + HALF[dtype] * 1.01 * np.abs(u) + 1e-30


def dx_bound(W, g, act, p, pre, dres, dx, dtype):
    d = g @ W
    dd = sum_bound(g.shape[1], np.abs(g) @ np.abs(W), dtype)
    if act != "none":
        off = {"relu": 0.0}.get(act, 32 * U if dtype == "f32" else 1.2e-4)
        dd = 1.13 * dd + off * np.abs(d)
    dd = (dd + 3 * U * 1.13 * np.abs(d)) / (1 - p)
    if dres is not None:
        dd = dd + 2 * U * (np.abs(dx) + np.abs(dres))
    return dd + HALF[dtype] * 1.01 * np.abs(dx) + 1e-30


def check_forward(lib, R, K, N, dtype, act="none", p=0.0, bias=True, res=False, pre=False, inplace=False, seed=0,
                  prepared=None):
    rng = np.random.default_rng(seed)
    x, W = tensor(rng, (R, K), dtype, 1.0, 0.25), tensor(rng, (N, K), dtype, 1.5 / np.sqrt(K))
    b = tensor(rng, (N,), "f32") if bias else None
    r = tensor(rng, (R, N), dtype) if res else None
    s = lib.make_linear(R, K, N, DTYPES[dtype])
    y, t0 = spare((R, N), DTYPES[dtype])
    q, t1 = spare((R, N), DTYPES[dtype])
    ws = lib.linear_workspace(s)
    wide = torch.cat([ws, torch.full((64,), 7, dtype=torch.uint8, device="cuda")])
    rnd = lib.dropout_rng(SEED, STEP) if p else None
    r_host = host(r)
    if inplace:
        y.copy_(r)
    lib.fs_linear_fwd(s, x, W, b, ACTS.index(act), p, rnd, y if inplace else r, y, q if pre else None, wide[:ws.numel()])
    torch.cuda.synchronize()
    assert untouched(t0, t1, wide[ws.numel():]) and (pre or untouched(q))
    assert int(wide[:4].view(torch.int32)[0]) == 0
    want, u = orc.linear(host(x), host(W), host(b), act, p, SEED, STEP, r_host)
    by, bu = forward_bound(host(x), host(W), host(b), act, p, r_host, want, u, dtype)
    off = np.abs(host(y) - want)
    assert (off <= by).all(), (np.argwhere(~(off <= by))[:4], (off / by).max())
    if pre:
        assert (np.abs(host(q) - u) <= bu).all()
    return y


def check_backward(lib, R, K, N, dtype, act="none", p=0.0, dres=False, accumulate=False, inplace=False, want_dx=True,
                   want_dw=True, want_db=True, seed=0):
    rng = np.random.default_rng(1000 + seed)
    x, W = tensor(rng, (R, K), dtype, 1.0, 0.25), tensor(rng, (N, K), dtype, 1.5 / np.sqrt(K))
    g = tensor(rng, (R, N), dtype)
    pre = tensor(rng, (R, K), dtype, 1.5) if act != "none" else None
    r = tensor(rng, (R, K), dtype) if dres else None
    s = lib.make_linear(R, K, N, DTYPES[dtype])
    dx, t0 = spare((R, K), DTYPES[dtype])
    dW, t1 = spare((N, K), torch.float32)
    db, t2 = spare((N,), torch.float32)
    ws = lib.linear_workspace(s, backward=True)
    wide = torch.cat([ws, torch.full((64,), 7, dtype=torch.uint8, device="cuda")])
    old_w, old_b = np.zeros((N, K)), np.zeros(N)
    if accumulate:
        dW.copy_(tensor(rng, (N, K), "f32"))
        db.copy_(tensor(rng, (N,), "f32"))
        old_w, old_b = host(dW), host(db)
    rnd = lib.dropout_rng(SEED, STEP) if p else None
    r_host = host(r)
    if inplace:
        dx.copy_(r)
    lib.fs_linear_bwd(s, x if want_dw else None, W if want_dx else None, g, ACTS.index(act), p, rnd, pre,
                      (dx if inplace else r) if want_dx else None, dx if want_dx else None, dW if want_dw else None,
                      db if want_db and want_dw else None, accumulate, wide[:ws.numel()])
    torch.cuda.synchronize()
    assert untouched(t0, t1, t2, wide[ws.numel():])
    assert int(wide[:4].view(torch.int32)[0]) == 0
    want, ww, wb = orc.linear_bwd(host(x), host(W), host(g), act, p, SEED, STEP, host(pre), r_host)
    if want_dx:
        bx = dx_bound(host(W), host(g), act, p, host(pre), r_host, want, dtype)
        off = np.abs(host(dx) - want)
        assert (off <= bx).all(), (np.argwhere(~(off <= bx))[:4], (off / bx).max())
    else:
        assert untouched(dx)
    if want_dw:
        bw = sum_bound(R, np.abs(host(g)).T @ np.abs(host(x)), "f32") + 2 * U * np.abs(ww + old_w)
        off = np.abs(host(dW) - (ww + old_w))
        assert (off <= bw).all(), (np.argwhere(~(off <= bw))[:4], (off / bw).max())
    if want_dw and want_db:
        bb = sum_bound(R, np.abs(host(g)).sum(0), "f32") + 2 * U * np.abs(wb + old_b)
        assert (np.abs(host(db) - (wb + old_b)) <= bb).all()
    elif not want_dw:
        assert untouched(dW, db)
