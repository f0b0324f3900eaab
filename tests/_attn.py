"""Cases of the token attention and the bounds that its results are held to.

u = 2^-24.  A product of two split operands drops at most 2^-22 = 4 u of itself (lo lo') and the
tf32 cut of the low parts costs as much again for each operand; a chain of n tensor-core steps
rounds its fp32 accumulator n times, at most 2 u of the terms' magnitudes each.  A score of d
channels is a chain of 3 d / 8 steps, a sum over n rows one of 3 n / 8 steps."""
import numpy as np
import torch

from oracle import operators_oracle as orc

U = 2.0 ** -24


def make(seed, B, H, Hkv, Gq, Gk, d, cap=0.0, bias=None, docs=0, prefix=None, bwd=True):
    """bias: None, "index" or "place"; docs: number of documents; prefix: None, 0 (no lengths given) or 1."""
    rng = np.random.default_rng(seed)

    def n(*s):
        return rng.standard_normal(s).astype(np.float32)

    c = {"B": B, "H": H, "Hkv": Hkv, "Gq": Gq, "Gk": Gk, "d": d, "cap": cap, "prefix": prefix, "scale": d ** -0.5,
         "q": n(B, H, Gq, d), "k": n(B, Hkv, Gk, d), "v": n(B, Hkv, Gk, d), "dout": n(B, H, Gq, d) if bwd else None}
    m = dict.fromkeys(("slopes", "pos_q", "pos_k", "doc_q", "doc_k", "prefix"))
    if bias:
        m["slopes"] = (0.3 * rng.random(H)).astype(np.float32)
    if bias == "place":
        m["pos_q"], m["pos_k"] = (10 * rng.random((B, Gq))).astype(np.float32), (10 * rng.random((B, Gk))).astype(np.float32)
    if docs:
        m["doc_k"] = rng.integers(-1, docs, (B, Gk)).astype(np.int32)
        m["doc_q"] = rng.integers(-1, docs + 1, (B, Gq)).astype(np.int32)  # one that no key has
    if prefix:
        m["prefix"] = rng.integers(0, Gk + 1, B).astype(np.int32)
    c["mask"] = m
    return c


def shape_of(lib, c):
    return lib.make_attn_shape(c["B"], c["H"], c["Gq"], c["d"], Hkv=c["Hkv"], Gk=c["Gk"], scale=c["scale"],
                               cap=c["cap"], prefix=c["prefix"] is not None)


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def mask_of(lib, c):
    return lib.attn_mask(**{k: dev(v) for k, v in c["mask"].items()})


def spare(shape, extra=64):
    n = int(np.prod(shape))
    buf = torch.full((n + extra,), 7.0, device="cuda")
    return buf[:n].view(shape), buf[n:]


def run(lib, c, stream=None, mask=None):
    """Forward, and the backward where the case has dout: numpy results."""
    s, m = shape_of(lib, c), mask or mask_of(lib, c)
    q, k, v = dev(c["q"]), dev(c["k"]), dev(c["v"])
    out, t0 = spare(q.shape)
    lse, t1 = spare(q.shape[:-1])
    ws = lib.attn_workspace(s)
    lib.fs_attn_fwd(s, q, k, v, m, out, lse, ws, stream=stream)
    assert lib.fs_device_status(ws, stream) == lib.FS_OK
    got, tails = {"out": out, "lse": lse}, [t0, t1]
    if c["dout"] is not None:
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            got[name], t = spare(like.shape)
            tails.append(t)
        ws = lib.attn_workspace(s, backward=True)
        lib.fs_attn_bwd(s, q, k, v, m, out, lse, dev(c["dout"]), got["dq"], got["dk"], got["dv"], ws, stream=stream)
        assert lib.fs_device_status(ws, stream) == lib.FS_OK
    assert all(bool((t == 7).all()) for t in tails)
    return {name: t.cpu().numpy() for name, t in got.items()}


def want(c):
    r = orc.attention(c["q"], c["k"], c["v"], c["scale"], c["cap"], dout=c["dout"],
                      **{n: t for n, t in c["mask"].items() if n != "prefix"},
                      prefix=None if c["prefix"] is None else
                      (c["mask"]["prefix"] if c["prefix"] else np.zeros(c["B"], np.int32)))
    return dict(zip(("out", "lse", "dq", "dk", "dv"), r))


def bounds(c, ref):
    """Elementwise bounds on the error of every result."""
    B, H, Hkv, Gq, Gk, d = (c[n] for n in ("B", "H", "Hkv", "Gq", "Gk", "d"))
    m, rep, rows = c["mask"], H // Hkv, (H // Hkv) * Gq
    tol = {n: np.zeros(r.shape) for n, r in ref.items()}
    # the magnitudes that a result is summed from: dout.v and D cancel in the score gradients
    # (wholly where a query sees one key), and rounding errors are relative to them
    mag_of = {n: np.abs(np.where(np.isfinite(r), r, 0)) for n, r in ref.items()}
    eps_d = (12 + 6 * d / 8) * U       # of the sum of a product's magnitudes over d channels
    eps_k = (12 + 6 * Gk / 8 + 64) * U  # over the keys (and joins of splits)
    eps_r = (12 + 6 * rows / 8 + 64) * U
    for b in range(B):
        ok = orc.visible(Gq, Gk, None if m["doc_q"] is None else m["doc_q"][b],
                         None if m["doc_k"] is None else m["doc_k"][b],
                         None if c["prefix"] is None else (m["prefix"][b] if c["prefix"] else 0))
        for h in range(H):
            q, k, v = (np.asarray(c[n][b, i], np.float64) for n, i in (("q", h), ("k", h // rep), ("v", h // rep)))
            s, mag = c["scale"] * q @ k.T, abs(c["scale"]) * np.abs(q) @ np.abs(k).T
            t = np.tanh(s / c["cap"]) if c["cap"] else np.zeros_like(s)
            a = c["cap"] * t if c["cap"] else s
            far = np.zeros_like(s)
            if m["slopes"] is not None:
                pq = np.arange(Gq) + Gk - Gq if m["pos_q"] is None else m["pos_q"][b].astype(np.float64)
                pk = np.arange(Gk) if m["pos_k"] is None else m["pos_k"][b].astype(np.float64)
                far = m["slopes"][h] * np.abs(pq[:, None] - pk[None, :])
                a = a - far
            with np.errstate(all="ignore"):
                lse = ref["lse"][b, h][:, None]
                p = np.where(ok & np.isfinite(lse), np.exp(a - lse), 0.0)
            # the score's error: the product's, then five roundings of the score, the cap and the
            # bias; tanhf's two units in the last place
            ds_ = eps_d * mag + 8 * U * (np.abs(s) + np.abs(a) + far + c["cap"] * np.abs(t))
            worst = np.where(ok, ds_, 0).max(1, keepdims=True)
            # a weight's: its score's, the statistic's (the largest score error, the sum's rounding
            # and its own rounding in each direction), two units of the exponential
            with np.errstate(invalid="ignore"):
                big = np.where(np.isfinite(lse), np.abs(lse), 0.0)
            dp_ = ds_ + worst + eps_k + (8 + 6 * big) * U
            tol["lse"][b, h] = (worst + eps_k + (8 + 4 * big) * U)[:, 0]
            tol["out"][b, h] = (p * (dp_ + eps_k)) @ np.abs(v) + 1e-30
            if c["dout"] is None:
                continue
            g = np.asarray(c["dout"][b, h], np.float64)
            D, dm = (g * ref["out"][b, h]).sum(1, keepdims=True), np.abs(g) @ np.abs(v).T
            dD = (tol["out"][b, h] * np.abs(g)).sum(1, keepdims=True) + d * U * np.abs(g * ref["out"][b, h]).sum(1, keepdims=True)
            dw = g @ v.T - D
            slope = c["scale"] * (1 - t * t)
            err = p * (np.abs(slope * dw) * (dp_ + 6 * U) + abs(c["scale"]) * np.abs(dw) * (8 * U + (2 * ds_ / c["cap"] if c["cap"] else 0))
                       + np.abs(slope) * (eps_d * dm + dD + 2 * U * (np.abs(dw) + np.abs(D))))
            ds = np.abs(p * slope * dw)
            whole = p * np.abs(slope) * (dm + np.abs(D))
            mag_of["dq"][b, h] = whole @ np.abs(k)
            mag_of["dk"][b, h // rep] += whole.T @ np.abs(q)
            tol["dq"][b, h] = err @ np.abs(k) + eps_k * ds @ np.abs(k) + 1e-30
            tol["dk"][b, h // rep] += err.T @ np.abs(q) + eps_r * ds.T @ np.abs(q) + 1e-30
            tol["dv"][b, h // rep] += (p * (dp_ + eps_r)).T @ np.abs(g) + 1e-30
    return tol, mag_of


def check(lib, c, got=None):
    got, ref = run(lib, c) if got is None else got, want(c)
    tol, mag = bounds(c, ref)
    for n, r in ref.items():
        fine = np.isfinite(r)
        assert np.array_equal(np.isfinite(got[n]), fine), n
        assert np.array_equal(got[n][~fine], r[~fine]), n
        off = np.abs(got[n][fine] - r[fine])
        over = off / tol[n][fine]
        assert (over <= 1).all(), f"{n}: {over.max():.3g} times its bound"
        # Roundings of either sign, of fp32's own order, stay far below the sum of their bounds.  But a
        # weight is 2^x with x = s f - lse log2(e), and an exponent's error is its relative error times ln 2:
        # the roundings of the factor f, of lse, of its product and of x are u of numbers up to |lse| log2(e)
        # (and 24 more: smaller weights do not count), all of one sign for a row or for the whole call.
        norm = np.linalg.norm(mag[n][fine])
        lse = np.abs(ref["lse"][np.isfinite(ref["lse"])]).max(initial=0.0)
        rel = 3e-6 + 4 * np.log(2) * U * (lse * np.log2(np.e) + 24)
        assert np.linalg.norm(off) <= rel * norm + 1e-30, f"{n}: {np.linalg.norm(off):.3g} off, terms of {norm:.3g}"
    return got
