"""The operators around the coupling, as cases that can be timed and compared.

  attn_fwd, attn_bwd   self-attention of the slice tokens, the token operation of the original
                       Transolver layer in place of the constant mix: scores with an optional
                       tanh cap, distance bias, document mask and prefix mask, shared key and
                       value heads (fs_attn_fwd, fs_attn_bwd)
  norm_fwd, norm_bwd   layer norm of the point features before a coupling, with the residual
                       stream's sum and an 8-bit checkpoint of it (fs_norm_fwd, fs_norm_bwd)
  ckpt                 an activation packed into 8 bits in the forward pass and restored in the
                       backward pass (fs_ckpt_pack, fs_ckpt_unpack)

`run` computes them in plain torch operations, or through the library where `own` is true.
"""
import math

import torch

own = False

BLOCK = 32  # channels that share a checkpoint's scale
EPS = 1e-5


# ---- cases -----------------------------------------------------------------------------------


def _attn(kind, B, H, Hkv, Gq, Gk, d, cap=0.0, bias=False, docs=0, prefix=False):
    return {"kind": kind, "B": B, "H": H, "Hkv": Hkv, "Gq": Gq, "Gk": Gk, "d": d, "cap": cap, "bias": bias,
            "docs": docs, "prefix": prefix}


def _rows(kind, rows, C, dtype, res=False, ckpt=False):
    return {"kind": kind, "rows": rows, "C": C, "dtype": dtype, "res": res, "ckpt": ckpt}


def listed():
    return [
        # The tokens of one small mesh at the usual slice count: the smallest call, latency.
        {"name": "attn_fwd_tiny", **_attn("attn_fwd", 1, 8, 8, 32, 32, 32)},
        # One query token per sample and head against all tokens of the largest slice count: a
        # probe of the state, work split over the keys.
        {"name": "attn_fwd_probe", **_attn("attn_fwd", 4, 8, 2, 1, 4096, 32, cap=20.0)},
        # Inference of the million-point mesh: 1024 slices, scores biased by distance.
        {"name": "attn_fwd_large_g", **_attn("attn_fwd", 1, 8, 8, 1024, 1024, 32, bias=True)},
        # A training step's backward on a surface mesh: odd slice count, wide shared heads.
        {"name": "attn_bwd_ragged", **_attn("attn_bwd", 3, 4, 2, 100, 100, 64, cap=20.0)},
        # The large training step: two samples of 512 slices, several bodies' tokens in a sample.
        {"name": "attn_bwd_train", **_attn("attn_bwd", 2, 8, 8, 512, 512, 32, cap=30.0, docs=3)},
        # The largest slice count, tokens of later time steps see the earlier ones only.
        {"name": "attn_bwd_prefix", **_attn("attn_bwd", 2, 8, 8, 4096, 4096, 32, bias=True, prefix=True)},
        # Norms of a small fp32 sample's tokens, head by head: latency.
        {"name": "norm_fwd_tokens", **_rows("norm_fwd", 256, 32, "f32")},
        # The features of the million-point mesh: residual sum, norm and checkpoint.
        {"name": "norm_fwd_large", **_rows("norm_fwd", 1048576, 256, "bf16", res=True, ckpt=True)},
        # An fp32 training sample of an odd number of points, widths off the vector size.
        {"name": "norm_bwd_ragged", **_rows("norm_bwd", 60033, 198, "f32")},
        # The large training step's norm: backward from the checkpoint, residual gradient added.
        {"name": "norm_bwd_large", **_rows("norm_bwd", 1048576, 256, "bf16", res=True, ckpt=True)},
        # A surface mesh's x_mid and fx of a few layers, fp32.
        {"name": "ckpt_surface", **_rows("ckpt", 32768, 256, "f32")},
        # The million-point mesh's x_mid.
        {"name": "ckpt_large", **_rows("ckpt", 1048576, 256, "bf16")},
    ]


def draw(rng):
    """Slice counts from 16 to 4096, rows from some hundred to a million, widths of 16 to 1024
    channels; odd sizes among all of them."""

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("attn_fwd", "attn_bwd", "attn_fwd", "attn_bwd", "norm_fwd", "norm_bwd", "ckpt"))
    if kind.startswith("attn"):
        while True:
            B, d = rng.choice((1, 1, 2, 3, 4)), rng.choice((32, 32, 16, 64))
            H = {16: 8, 32: 8, 64: 4}[d]
            Hkv = H // rng.choice((1, 1, 2, 4))
            Gk = log(16, 4096)
            if rng.random() < 0.4:  # the usual slice counts
                Gk = 1 << round(math.log2(Gk))
            Gq = Gk if kind == "attn_bwd" or rng.random() < 0.75 else rng.randint(1, min(16, Gk))
            c = _attn(kind, B, H, Hkv, Gq, Gk, d, rng.choice((0.0, 0.0, 20.0, 30.0)), rng.random() < 0.4,
                      rng.choice((0, 0, 2, 5)), rng.random() < 0.3)
            if B * H * Gq * Gk * d <= 2 * 8 * 4096 * 4096 * 32 // (1 if kind == "attn_bwd" else 2):
                return c
    while True:
        rows = log(200, 1 << 20)
        C = rng.choice((256, 256, log(16, 1024), 8 * log(2, 128)))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        ckpt = kind != "ckpt" and rng.random() < 0.5
        res = kind != "ckpt" and rng.random() < 0.5
        if rows * C * (2 if dtype == "f32" else 1) <= 1 << 28:
            return _rows(kind, rows, C, dtype, res, ckpt)


# ---- inputs ----------------------------------------------------------------------------------


def _bounds(G, docs):
    """First token of each document but the first: documents of unequal lengths."""
    return [int(G * ((k + 1) / docs) ** 1.4) for k in range(docs - 1)]


def _prefixes(c):
    return [c["Gk"] * (b + 1) // (4 * c["B"]) for b in range(c["B"])]


def _attn_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, H, Hkv, Gq, Gk, d = (c[k] for k in ("B", "H", "Hkv", "Gq", "Gk", "d"))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # Projected tokens: unit variance, with a part that the tokens of a head share.
    v = {"q": normal(B, H, Gq, d) + 0.5 * normal(B, H, 1, d), "k": normal(B, Hkv, Gk, d) + 0.5 * normal(B, Hkv, 1, d),
         "v": normal(B, Hkv, Gk, d), "slopes": None, "pos_q": None, "pos_k": None, "doc_q": None, "doc_k": None,
         "prefix": None}
    if c["bias"]:  # a decay per head, and each token's place along the body
        v["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H)
        place = torch.sort(torch.rand(B, Gk, generator=g, device="cuda"), dim=1).values * 100.0
        v["pos_k"] = place
        v["pos_q"] = place[:, Gk - Gq:].contiguous()
    if c["docs"]:  # the body a token belongs to; a few slots of each sample are unused
        doc = torch.bucketize(torch.arange(Gk, device="cuda"),
                              torch.tensor(_bounds(Gk, c["docs"]), device="cuda"), right=True).expand(B, Gk)
        dead = torch.rand(B, Gk, generator=g, device="cuda") < 0.03
        doc = torch.where(dead, torch.full_like(doc, -1), doc).to(torch.int32)
        v["doc_k"] = doc.contiguous()
        v["doc_q"] = doc[:, Gk - Gq:].contiguous()
    if c["prefix"]:
        v["prefix"] = torch.tensor(_prefixes(c), dtype=torch.int32, device="cuda")
    if c["kind"] == "attn_bwd":
        v["dout"] = normal(B, H, Gq, d)
        v["out"], v["lse"], _, _ = _attn_plain(c, v)
    return v


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _rows_inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    R, C, dt = c["rows"], c["C"], _dtype(c)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)

    # Hidden features: channels of different sizes and offsets, a few large ones.
    size = torch.exp(0.5 * normal(C)).to(dt)
    v = {"x": torch.addcmul(normal(C).to(dt), normal(R, C, dtype=dt), size)}
    if c["kind"] == "ckpt":
        return v
    v["gamma"] = 1.0 + 0.2 * normal(C)
    v["beta"] = 0.2 * normal(C)
    if c["kind"] == "norm_fwd":
        v["res"] = normal(R, C, dtype=dt) if c["res"] else None
        return v
    f = v["x"].float()
    v["mean"] = f.mean(1)
    v["rstd"] = torch.rsqrt(f.var(1, unbiased=False) + EPS)
    v["dy"] = normal(R, C, dtype=dt)
    v["dres"] = normal(R, C, dtype=dt) if c["res"] else None
    if c["ckpt"]:
        v["q8"], v["e8"] = _pack_plain(v.pop("x"))
    return v


def prepare(case, seed):
    """Inputs, and the buffers and scratch that a program keeps for its layers."""
    c = case
    if c["kind"].startswith("attn"):
        v = _attn_inputs(c, seed)
        s = {"case": c, "in": v}
        if own:
            from paper_2609_32525_gb300 import flashslice as fs

            bwd = c["kind"] == "attn_bwd"
            s["shape"] = fs.make_attn_shape(c["B"], c["H"], c["Gq"], c["d"], Hkv=c["Hkv"], Gk=c["Gk"], cap=c["cap"],
                                            prefix=c["prefix"])
            s["mask"] = fs.attn_mask(*(v[k] for k in ("slopes", "pos_q", "pos_k", "doc_q", "doc_k", "prefix")))
            s["ws"] = fs.attn_workspace(s["shape"], backward=bwd)
            if bwd:
                s["out"] = {"dq": torch.empty_like(v["q"]), "dk": torch.empty_like(v["k"]),
                            "dv": torch.empty_like(v["v"])}
            else:
                s["out"] = {"out": torch.empty_like(v["q"]), "lse": torch.empty_like(v["q"][..., 0])}
        return s
    v = _rows_inputs(c, seed)
    s = {"case": c, "in": v}
    if own:
        from paper_2609_32525_gb300 import flashslice as fs

        R, C, dt = c["rows"], c["C"], _dtype(c)
        s["rows"] = fs.make_rows(R, C, dt)
        s["packed"] = fs.checkpoint(s["rows"]) if c["ckpt"] or c["kind"] == "ckpt" else (None, None)
        if c["kind"] == "ckpt":
            s["out"] = {"x": torch.empty_like(v["x"])}
        elif c["kind"] == "norm_fwd":
            s["out"] = {"y": torch.empty_like(v["x"]), "mean": torch.empty(R, device="cuda"),
                        "rstd": torch.empty(R, device="cuda"), "sum": torch.empty_like(v["x"]) if c["res"] else None,
                        "kept": torch.empty_like(v["x"]) if c["ckpt"] else None}
        else:
            s["ws"] = fs.norm_workspace(s["rows"])
            s["out"] = {"dx": torch.empty_like(v["dy"]), "dgamma": torch.empty_like(v["gamma"]),
                        "dbeta": torch.empty_like(v["beta"])}
    return s


# ---- the plain forms ---------------------------------------------------------------------------


def _visible(c, v):
    """[B, 1, Gq, Gk]: which keys a query sees; None where it sees all."""
    ok = None
    if v["doc_q"] is not None:
        ok = ((v["doc_q"][:, :, None] == v["doc_k"][:, None, :]) & (v["doc_k"] >= 0)[:, None, :])[:, None]
    if v["prefix"] is not None:
        i = torch.arange(c["Gq"], device="cuda") + (c["Gk"] - c["Gq"])
        j = torch.arange(c["Gk"], device="cuda")
        see = (j[None, :] <= i[:, None])[None] | (j[None, None, :] < v["prefix"][:, None, None])
        ok = see[:, None] if ok is None else ok & see[:, None]
    return ok


def _attn_plain(c, v):
    """out, lse, and for the backward the probabilities and the cap's derivative."""
    B, H, Hkv, Gq, Gk, d = (c[k] for k in ("B", "H", "Hkv", "Gq", "Gk", "d"))
    k = v["k"].repeat_interleave(H // Hkv, dim=1)
    s = (v["q"] @ k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    slope = None
    if c["cap"]:
        t = torch.tanh(s / c["cap"])
        s, slope = c["cap"] * t, 1.0 - t * t
    if v["slopes"] is not None:
        far = (v["pos_q"][:, :, None] - v["pos_k"][:, None, :]).abs()
        s = s - v["slopes"][None, :, None, None] * far[:, None]
    ok = _visible(c, v)
    if ok is not None:
        s = torch.where(ok, s, torch.full_like(s, -math.inf))
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    out = p @ v["v"].repeat_interleave(H // Hkv, dim=1)
    return out, (top + torch.log(total)).squeeze(-1), p, slope


def _attn_bwd_plain(c, v):
    B, H, Hkv, Gq, Gk, d = (c[k] for k in ("B", "H", "Hkv", "Gq", "Gk", "d"))
    _, _, p, slope = _attn_plain(c, v)
    k, val, do = v["k"].repeat_interleave(H // Hkv, dim=1), v["v"].repeat_interleave(H // Hkv, dim=1), v["dout"]
    ds = p * (do @ val.transpose(-1, -2) - (do * v["out"]).sum(-1, keepdim=True))
    if slope is not None:
        ds = ds * slope
    ds = ds * (1.0 / math.sqrt(d))
    shared = (B, Hkv, H // Hkv, Gk, d)
    return {"dq": ds @ k, "dk": (ds.transpose(-1, -2) @ v["q"]).view(shared).sum(2),
            "dv": (p.transpose(-1, -2) @ do).view(shared).sum(2)}


def _power(e):
    """2 ** e in fp32 for whole e in [-126, 127]."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _pack_plain(x):
    """8-bit values and the byte s + 127 of each block's scale 2 ** s: the smallest s that
    brings the block's largest magnitude to at most 127; 255 for a block with NaN or infinity."""
    R, C = x.shape
    f = torch.nn.functional.pad(x.float(), (0, -C % BLOCK)).view(R, -1, BLOCK)
    top = f.abs().amax(-1)
    fine = top < math.inf
    top = torch.where(fine, top, torch.ones_like(top))
    s = (torch.frexp(top).exponent - 7).clamp(-126, 127)
    s = s + (torch.round(top * _power(-s)) > 127).int()
    q = torch.round(torch.where(fine[..., None], f, torch.zeros_like(f)) * _power(-s)[..., None])
    e = torch.where(fine, s + 127, torch.full_like(s, 255))
    return q.view(R, -1)[:, :C].to(torch.int8).contiguous(), e.to(torch.uint8).contiguous()


def _unpack_plain(q8, e8, dtype):
    e = e8.int()
    size = torch.where(e < 255, _power(torch.where(e < 255, e, torch.full_like(e, 127)) - 127),
                       torch.full_like(e, math.nan, dtype=torch.float32))
    return (q8.float() * size.repeat_interleave(BLOCK, dim=1)[:, :q8.shape[1]]).to(dtype)


def _norm_fwd_plain(c, v):
    x, dt = v["x"], _dtype(c)
    if v["res"] is not None:
        x = (x.float() + v["res"].float()).to(dt)
    f = x.float()
    mean = f.mean(1)
    f = f - mean[:, None]
    rstd = 1.0 / torch.sqrt((f * f).mean(1) + EPS)
    out = {"y": (f * rstd[:, None] * v["gamma"] + v["beta"]).to(dt), "mean": mean, "rstd": rstd}
    if v["res"] is not None:
        out["sum"] = x
    if c["ckpt"]:
        out["kept"] = _unpack_plain(*_pack_plain(x), dt)
    return out


def _norm_bwd_plain(c, v):
    x = (_unpack_plain(v["q8"], v["e8"], torch.float32) if c["ckpt"] else v["x"].float())
    xh = (x - v["mean"][:, None]) * v["rstd"][:, None]
    dy = v["dy"].float()
    g = dy * v["gamma"]
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * v["rstd"][:, None]
    if v["dres"] is not None:
        dx = dx + v["dres"].float()
    return {"dx": dx.to(_dtype(c)), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}


def _run_own(state):
    from paper_2609_32525_gb300 import flashslice as fs

    c, v, o = state["case"], state["in"], state["out"]
    kind = c["kind"]
    if kind == "attn_fwd":
        fs.fs_attn_fwd(state["shape"], v["q"], v["k"], v["v"], state["mask"], o["out"], o["lse"], state["ws"])
        return o
    if kind == "attn_bwd":
        fs.fs_attn_bwd(state["shape"], v["q"], v["k"], v["v"], state["mask"], v["out"], v["lse"], v["dout"], o["dq"],
                       o["dk"], o["dv"], state["ws"])
        return o
    q8, e8 = state["packed"]
    if kind == "ckpt":
        fs.fs_ckpt_pack(state["rows"], v["x"], q8, e8)
        fs.fs_ckpt_unpack(state["rows"], q8, e8, o["x"])
        return o
    if kind == "norm_fwd":
        fs.fs_norm_fwd(state["rows"], v["x"], v["res"], v["gamma"], v["beta"], EPS, o["sum"], o["y"], o["mean"],
                       o["rstd"], q8, e8)
        if c["ckpt"]:
            fs.fs_ckpt_unpack(state["rows"], q8, e8, o["kept"])
        return o
    fs.fs_norm_bwd(state["rows"], v.get("x"), v.get("q8"), v.get("e8"), v["gamma"], v["mean"], v["rstd"], v["dy"],
                   v["dres"], o["dx"], o["dgamma"], o["dbeta"], False, state["ws"])
    return o


def run(state):
    if own:
        return _run_own(state)
    c, v = state["case"], state["in"]
    if c["kind"] == "attn_fwd":
        out, lse, _, _ = _attn_plain(c, v)
        return {"out": out, "lse": lse}
    if c["kind"] == "attn_bwd":
        return _attn_bwd_plain(c, v)
    if c["kind"] == "ckpt":
        return {"x": _unpack_plain(*_pack_plain(v["x"]), _dtype(c))}
    return _norm_fwd_plain(c, v) if c["kind"] == "norm_fwd" else _norm_bwd_plain(c, v)


# ---- what a pass cannot do without -------------------------------------------------------------


def _pairs(c):
    """(query, key) pairs that the masks leave, per head, over the batch."""
    Gq, Gk, B = c["Gq"], c["Gk"], c["B"]
    off = Gk - Gq
    cuts = [0] + (_bounds(Gk, c["docs"]) if c["docs"] else []) + [Gk]
    total = 0
    for b in range(B):
        pre = _prefixes(c)[b]
        for lo, hi in zip(cuts, cuts[1:]):
            for i in range(max(lo, off), hi):
                total += hi - lo if not c["prefix"] else max(0, min(hi, max(i + 1, pre)) - lo)
    return total


def work(case):
    c = case
    if c["kind"].startswith("attn"):
        q, kv = c["B"] * c["H"] * c["Gq"] * c["d"], c["B"] * c["Hkv"] * c["Gk"] * c["d"]
        stat = c["B"] * c["H"] * c["Gq"]
        places = c["B"] * (c["Gq"] + c["Gk"]) * ((1 if c["bias"] else 0) + (1 if c["docs"] else 0))
        flops = 2 * c["H"] * _pairs(c) * c["d"]
        if c["kind"] == "attn_fwd":
            return {"bytes": 4 * (2 * q + 2 * kv + stat + places), "flops": 2 * flops}
        return {"bytes": 4 * (4 * q + 4 * kv + stat + places), "flops": 5 * flops}
    n, R, C = c["rows"] * c["C"], c["rows"], c["C"]
    e = 2 if c["dtype"] == "bf16" else 4
    packed = n + R * ((C + BLOCK - 1) // BLOCK)
    if c["kind"] == "ckpt":
        return {"bytes": 2 * n * e + 2 * packed, "flops": 4 * n}
    if c["kind"] == "norm_fwd":  # the checkpoint is written, and read back into the values it stands for
        return {"bytes": n * e * (4 if c["res"] else 2) + (2 * packed + n * e if c["ckpt"] else 0) + 8 * R + 8 * C,
                "flops": 8 * n}
    return {"bytes": n * e * (3 if c["res"] else 2) + (packed if c["ckpt"] else n * e) + 8 * R + 12 * C,
            "flops": 14 * n}


# ---- the same in 64 bits -------------------------------------------------------------------------


def _attn_exact(c, seed):
    if c["B"] * c["H"] * c["Gq"] * c["Gk"] * c["d"] > 1 << 34:
        return None
    v = _attn_inputs(c, seed)
    B, H, Hkv, Gq, Gk, d = (c[k] for k in ("B", "H", "Hkv", "Gq", "Gk", "d"))
    D = dict(dtype=torch.float64, device="cuda")
    bwd = c["kind"] == "attn_bwd"
    out, lse = torch.zeros(B, H, Gq, d, **D), torch.full((B, H, Gq), -math.inf, **D)
    dq, dk, dv = torch.zeros(B, H, Gq, d, **D), torch.zeros(B, Hkv, Gk, d, **D), torch.zeros(B, Hkv, Gk, d, **D)
    at = torch.arange(Gk - Gq, Gk, device="cuda")[:, None]
    to = torch.arange(Gk, device="cuda")[None, :]
    for b in range(B):
        hide = torch.zeros(Gq, Gk, dtype=torch.bool, device="cuda")
        if v["doc_q"] is not None:
            hide |= v["doc_q"][b][:, None] != v["doc_k"][b][None, :]
            hide |= (v["doc_k"][b] < 0)[None, :]
        if v["prefix"] is not None:
            hide |= (to > at) & (to >= v["prefix"][b])
        alive = ~hide.all(1)
        for h in range(H):
            kh = h * Hkv // H
            q, k, val = v["q"][b, h].double(), v["k"][b, kh].double(), v["v"][b, kh].double()
            raw = torch.einsum("ic,jc->ij", q, k) / math.sqrt(d)
            a = c["cap"] * torch.tanh(raw / c["cap"]) if c["cap"] else raw
            if v["slopes"] is not None:
                a = a - v["slopes"][h].double() * torch.cdist(v["pos_q"][b].double()[:, None],
                                                              v["pos_k"][b].double()[:, None])
            a = a.masked_fill(hide, -math.inf)[alive]
            z = torch.logsumexp(a, 1)
            lse[b, h, alive] = z
            w = torch.exp(a - z[:, None])
            o = torch.einsum("ij,jc->ic", w, val)
            out[b, h, alive] = o
            if bwd:
                g = v["dout"][b, h].double()[alive]
                dv[b, kh] += torch.einsum("ij,ic->jc", w, g)
                dw = torch.einsum("ic,jc->ij", g, val)
                da = w * (dw - (w * dw).sum(1, keepdim=True))
                if c["cap"]:
                    da = da / torch.cosh(raw[alive] / c["cap"]) ** 2
                da = da / math.sqrt(d)
                dq[b, h, alive] = da @ k
                dk[b, kh] += da.T @ q[alive]
    return {"dq": dq, "dk": dk, "dv": dv} if bwd else {"out": out, "lse": lse}


def _kept_exact(x):
    """The values that the 8-bit checkpoint of x stands for, block by block in 64 bits."""
    parts = []
    for col in range(0, x.shape[1], BLOCK):
        f = x[:, col:col + BLOCK].double()
        top = f.abs().amax(1, keepdim=True)
        step = torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=2.0 ** -120))) - 6)
        step = torch.where(torch.round(top / step) > 127, 2 * step, step)
        parts.append(torch.round(f / step) * step)
    return torch.cat(parts, 1)


def exact(case, seed):
    c = case
    if c["kind"].startswith("attn"):
        return _attn_exact(c, seed)
    v = _rows_inputs(c, seed)
    if c["kind"] == "ckpt":
        return {"x": _kept_exact(v["x"])}
    if c["kind"] == "norm_fwd":
        x = v["x"]
        if v["res"] is not None:  # the sum is kept in the inputs' type, and normalised as it is kept
            x = (x.double() + v["res"].double()).to(_dtype(c))
        f = x.double()
        var, mean = torch.var_mean(f, dim=1, correction=0)
        rstd = (var + EPS).pow(-0.5)
        y = torch.addcmul(v["beta"].double(), (f - mean[:, None]) * rstd[:, None], v["gamma"].double())
        out = {"y": y, "mean": mean, "rstd": rstd}
        if v["res"] is not None:
            out["sum"] = f
        if c["ckpt"]:
            out["kept"] = _kept_exact(x)
        return out
    if c["ckpt"]:
        sizes = torch.pow(2.0, v["e8"].double() - 127.0)
        x = v["q8"].double()
        for n in range(sizes.shape[1]):
            x[:, n * BLOCK:(n + 1) * BLOCK] *= sizes[:, n:n + 1]
    else:
        x = v["x"].double()
    rstd = v["rstd"].double()[:, None]
    xh = (x - v["mean"].double()[:, None]) * rstd
    dy = v["dy"].double()
    dgamma, dbeta = torch.einsum("rc,rc->c", dy, xh), dy.sum(0)
    a = dy * v["gamma"].double()
    dx = rstd * (a - (a.sum(1, keepdim=True) + xh * (a * xh).sum(1, keepdim=True)) / c["C"])
    if v["dres"] is not None:
        dx += v["dres"].double()
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
