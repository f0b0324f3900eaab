"""The layer's linear maps and its dropout, as cases that can be timed and compared.

  linear_fwd   y = res + drop(act(x W^T + bias)): the projections into and out of a coupling and
               the two halves of a layer's MLP, with the pre-activation kept where a backward
               pass needs it (fs_linear_fwd)
  linear_bwd   the gradients of x, W and bias; the gradient of x goes on through the activation
               and the dropout that made x, and takes in the residual stream's (fs_linear_bwd)
  drop_fwd, drop_bwd
               y = res + drop(act(x)) and its gradient; the mask comes from a counter-based
               generator and is never stored (fs_dropout_fwd, fs_dropout_bwd)

`run` computes them in plain torch operations, or through the library where `own` is true.
"""
import math

import torch

own = False

ACTS = ("none", "relu", "gelu", "silu")


# ---- cases -----------------------------------------------------------------------------------


def _linear(kind, rows, cin, cout, dtype, act="none", p=0.0, res=False, pre=False):
    return {"kind": kind, "rows": rows, "cin": cin, "cout": cout, "dtype": dtype, "act": act, "p": p, "res": res,
            "pre": pre}


def _drop(kind, rows, C, dtype, act="none", p=0.1, res=False):
    return {"kind": kind, "rows": rows, "cin": C, "cout": C, "dtype": dtype, "act": act, "p": p, "res": res,
            "pre": False}


def listed():
    return [
        # A single probe point through a wide MLP's first half: the weights are all there is to read.
        {"name": "linear_fwd_probe", **_linear("linear_fwd", 1, 1024, 4096, "bf16", "gelu")},
        # The tokens of one small mesh through a projection, fp32: latency.
        {"name": "linear_fwd_tokens", **_linear("linear_fwd", 256, 32, 32, "f32")},
        # The million-point mesh's projection out of the coupling in training: dropout and residual.
        {"name": "linear_fwd_large", **_linear("linear_fwd", 1048576, 256, 256, "bf16", p=0.1, res=True)},
        # A surface mesh through the first half of a wide MLP in training: arithmetic.
        {"name": "linear_fwd_wide", **_linear("linear_fwd", 32768, 1024, 4096, "bf16", "gelu", pre=True)},
        # An fp32 sample of an odd number of points, widths off the vector size.
        {"name": "linear_fwd_ragged", **_linear("linear_fwd", 60033, 198, 330, "f32", "silu", res=True)},
        # A small sample's backward of odd sizes: latency.
        {"name": "linear_bwd_small", **_linear("linear_bwd", 100, 64, 66, "bf16", "gelu")},
        # The large training step, first half of the MLP: the gradient joins the residual stream's.
        {"name": "linear_bwd_large", **_linear("linear_bwd", 1048576, 256, 256, "bf16", res=True)},
        # The surface mesh back through the second half of the wide MLP, activation and dropout.
        {"name": "linear_bwd_wide", **_linear("linear_bwd", 32768, 4096, 1024, "bf16", "gelu", p=0.1)},
        # An fp32 training step of a volume mesh.
        {"name": "linear_bwd_f32", **_linear("linear_bwd", 131072, 256, 256, "f32", "gelu")},
        # The tokens of one small mesh: latency.
        {"name": "drop_fwd_tokens", **_drop("drop_fwd", 256, 32, "f32")},
        # The million-point mesh's residual stream.
        {"name": "drop_fwd_large", **_drop("drop_fwd", 1048576, 256, "bf16", res=True)},
        # An odd number of points and channels, back through activation and dropout.
        {"name": "drop_bwd_ragged", **_drop("drop_bwd", 60033, 198, "f32", "gelu", 0.25)},
    ]


def draw(rng):
    """One row to a million, widths of 16 to 4096 channels, odd ones among them."""

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width():
        return rng.choice((256, log(16, 1024), 8 * log(2, 128), 64 * log(1, 64)))

    while True:
        kind = rng.choice(("linear_fwd", "linear_bwd", "linear_fwd", "linear_bwd", "linear_fwd", "linear_bwd",
                           "drop_fwd", "drop_bwd"))
        rows, cin, cout = log(1, 1 << 20), width(), width()
        dtype = rng.choice(("bf16", "bf16", "f32"))
        act = rng.choice(("none", "none", "gelu", "gelu", "relu", "silu"))
        p = rng.choice((0.0, 0.0, 0.1, 0.25))
        res = rng.random() < 0.4
        e = 4 if dtype == "f32" else 2
        if kind.startswith("drop"):
            if rows * cin * e <= 1 << 29:
                return _drop(kind, rows, cin, dtype, act, p or 0.5, res and kind == "drop_fwd")
        elif rows * cin * cout <= 1 << 37 and rows * (cin + cout) * e <= 1 << 30:
            return _linear(kind, rows, cin, cout, dtype, act, p, res,
                           kind == "linear_fwd" and act != "none" and rng.random() < 0.6)


# ---- inputs ----------------------------------------------------------------------------------


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    R, K, N, dt = c["rows"], c["cin"], c["cout"], _dtype(c)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)

    v = {"rng": None, "res": None, "pre": None}
    if c["p"]:  # the generator's seed, and the number of the step and place in the network
        v["rng"] = torch.randint(0, 1 << 62, (2,), generator=g, device="cuda")
    # Features after a norm: channels of different sizes and offsets.
    size = (0.3 * normal(K)).exp().to(dt)
    v["x"] = torch.addcmul((0.3 * normal(K)).to(dt), normal(R, K, dtype=dt), size)
    if c["kind"] == "drop_fwd":
        v["res"] = normal(R, K, dtype=dt) if c["res"] else None
        return v
    if c["kind"] == "drop_bwd":
        v["pre"], v["g"] = (v.pop("x") if c["act"] != "none" else None), normal(R, K, dtype=dt)
        return v
    v["W"] = (normal(N, K) / math.sqrt(K)).to(dt)
    if c["kind"] == "linear_fwd":
        v["bias"] = 0.2 * normal(N)
        v["res"] = normal(R, N, dtype=dt) if c["res"] else None
        return v
    v["g"] = normal(R, N, dtype=dt)
    v["res"] = normal(R, K, dtype=dt) if c["res"] else None
    if c["act"] != "none":  # x came from these
        v["pre"] = v["x"]
        v["x"] = _act(c, v["x"].float())[0].to(dt)
    return v


def prepare(case, seed):
    """Inputs, and the buffers and scratch that a program keeps for its layers."""
    c = case
    v = _inputs(c, seed)
    s = {"case": c, "in": v}
    if own:
        from paper_2609_32525_gb300 import flashslice as fs

        R, K, N, dt = c["rows"], c["cin"], c["cout"], _dtype(c)
        if c["kind"].startswith("drop"):
            s["rows"] = fs.make_rows(R, K, dt)
            s["out"] = {"y": torch.empty(R, K, dtype=dt, device="cuda")}
            return s
        s["linear"] = fs.make_linear(R, K, N, dt)
        s["ws"] = fs.linear_workspace(s["linear"], backward=c["kind"] == "linear_bwd")
        if c["kind"] == "linear_fwd":
            s["out"] = {"y": torch.empty(R, N, dtype=dt, device="cuda")}
            if c["pre"]:
                s["out"]["pre"] = torch.empty(R, N, dtype=dt, device="cuda")
        else:
            s["out"] = {"dx": torch.empty(R, K, dtype=dt, device="cuda"), "dW": torch.empty(N, K, device="cuda"),
                        "dbias": torch.empty(N, device="cuda")}
    return s


# ---- the plain forms ---------------------------------------------------------------------------


def _act(c, u):
    """act(u) and act'(u)."""
    if c["act"] == "relu":
        on = (u > 0).to(u.dtype)
        return u * on, on
    if c["act"] == "gelu":
        cdf = 0.5 * torch.special.erfc(u * -math.sqrt(0.5))
        return u * cdf, cdf + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
    if c["act"] == "silu":
        sig = 1.0 / (1.0 + torch.exp(-u))
        return u * sig, sig * (1.0 + u * (1.0 - sig))
    return u, None


LOW = 0xFFFFFFFF


def _words(c0, c1, c2, c3, k0, k1):
    """Philox 4x32-10 of the counters (c0, c1, c2, c3) under the key (k0, k1): int64 tensors of
    32-bit words (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3)."""
    for _ in range(10):
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # 64-bit products, modulo 2^64
        c0, c1, c2, c3 = (((q >> 32) & LOW) ^ c1 ^ k0, q & LOW, ((p >> 32) & LOW) ^ c3 ^ k1, p & LOW)
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return torch.stack((c0, c1, c2, c3), -1)


def _threshold(c):
    """A value is kept where its 32-bit word is at least this; p as the calls take it, in fp32."""
    return int(torch.tensor(c["p"], dtype=torch.float32).double().item() * 4294967296.0)


def _scale(c):
    return 1.0 / (1.0 - torch.tensor(c["p"], dtype=torch.float32).double().item())


def _keep(c, rng, a):
    """Dropout of a [R, C]: four channels of a row share a counter."""
    if not c["p"]:
        return a
    R, C = a.shape
    quads = (C + 3) // 4
    at = torch.arange(R * quads, device="cuda")
    seed, step = rng[0], rng[1]
    w = _words(at & LOW, at >> 32, (step & LOW).expand_as(at), ((step >> 32) & LOW).expand_as(at), seed & LOW,
               (seed >> 32) & LOW)
    kept = (w >= _threshold(c)).view(R, 4 * quads)[:, :C]
    return torch.where(kept, a * _scale(c), torch.zeros_like(a))


def _plain(c, v):
    dt = _dtype(c)
    res = None if v["res"] is None else v["res"].float()
    if c["kind"] == "linear_fwd":
        u = v["x"].float() @ v["W"].float().T + v["bias"]
        y = _keep(c, v["rng"], _act(c, u)[0])
        out = {"y": (y if res is None else y + res).to(dt)}
        if c["pre"]:
            out["pre"] = u.to(dt)
        return out
    if c["kind"] == "drop_fwd":
        y = _keep(c, v["rng"], _act(c, v["x"].float())[0])
        return {"y": (y if res is None else y + res).to(dt)}
    g = v["g"].float()
    d = g if c["kind"] == "drop_bwd" else g @ v["W"].float()
    if v["pre"] is not None:
        d = d * _act(c, v["pre"].float())[1]
    d = _keep(c, v["rng"], d)
    d = (d if res is None else d + res).to(dt)
    if c["kind"] == "drop_bwd":
        return {"y": d}
    return {"dx": d, "dW": g.T @ v["x"].float(), "dbias": g.sum(0)}


def _run_own(state):
    from paper_2609_32525_gb300 import flashslice as fs

    c, v, o = state["case"], state["in"], state["out"]
    act = ACTS.index(c["act"])
    if c["kind"] == "linear_fwd":
        fs.fs_linear_fwd(state["linear"], v["x"], v["W"], v["bias"], act, c["p"], v["rng"], v["res"], o["y"],
                         o.get("pre"), state["ws"])
    elif c["kind"] == "linear_bwd":
        fs.fs_linear_bwd(state["linear"], v["x"], v["W"], v["g"], act, c["p"], v["rng"], v["pre"], v["res"], o["dx"],
                         o["dW"], o["dbias"], False, state["ws"])
    elif c["kind"] == "drop_fwd":
        fs.fs_dropout_fwd(state["rows"], v["x"], act, c["p"], v["rng"], v["res"], o["y"])
    else:
        fs.fs_dropout_bwd(state["rows"], v["g"], act, c["p"], v["rng"], v["pre"], o["y"])
    return o


def run(state):
    if own:
        return _run_own(state)
    return _plain(state["case"], state["in"])


# ---- what a pass cannot do without -------------------------------------------------------------


def work(case):
    c = case
    R, K, N = c["rows"], c["cin"], c["cout"]
    e = 2 if c["dtype"] == "bf16" else 4
    act = 1 if c["act"] != "none" else 0
    if c["kind"] == "drop_fwd":
        return {"bytes": R * K * e * (3 if c["res"] else 2), "flops": 4 * R * K}
    if c["kind"] == "drop_bwd":
        return {"bytes": R * K * e * (2 + act), "flops": 4 * R * K}
    if c["kind"] == "linear_fwd":
        return {"bytes": e * (R * K + N * K + R * N * (1 + c["res"] + c["pre"])) + 4 * N, "flops": 2 * R * K * N}
    return {"bytes": e * (R * K * (2 + act + c["res"]) + R * N + N * K) + 4 * (N * K + N), "flops": 4 * R * K * N}


# ---- the same in 64 bits -------------------------------------------------------------------------


def _times(a, m):
    """High and low 32 bits of the products of 32-bit words a with the 32-bit constant m, in
    products of halves."""
    lo, hi = (a & 0xFFFF) * m, (a >> 16) * m
    hi = hi + (lo >> 16)
    return hi >> 16, ((hi & 0xFFFF) << 16) | (lo & 0xFFFF)


def _kept_exact(c, rng, R, C):
    """[R, C] of truth values: what the dropout keeps."""
    seed, step = (int(t) for t in rng.tolist())
    row = torch.arange(R, device="cuda")[:, None]
    n = row * (-(-C // 4)) + torch.arange(-(-C // 4), device="cuda")[None, :]
    x = [n % (1 << 32), torch.div(n, 1 << 32, rounding_mode="floor"), torch.full_like(n, step % (1 << 32)),
         torch.full_like(n, step >> 32)]
    for i in range(10):
        key = ((seed + i * 0x9E3779B9) % (1 << 32), ((seed >> 32) + i * 0xBB67AE85) % (1 << 32))
        h0, l0 = _times(x[0], 0xD2511F53)
        h1, l1 = _times(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0]
    out = torch.empty(R, n.shape[1], 4, dtype=torch.bool, device="cuda")
    for j in range(4):
        out[..., j] = x[j].double() / 4294967296.0 >= _threshold(c) / 4294967296.0
    return out.flatten(1)[:, :C]


def _act_exact(c, u):
    if c["act"] == "relu":
        return torch.clamp(u, min=0.0)
    if c["act"] == "gelu":
        return u * torch.special.ndtr(u)
    if c["act"] == "silu":
        return u * torch.sigmoid(u)
    return u


def _slope_exact(c, u):
    if c["act"] == "relu":
        return torch.heaviside(u, torch.zeros((), dtype=u.dtype, device=u.device))
    if c["act"] == "gelu":
        return torch.special.ndtr(u) + u * torch.exp(-u.square() / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(u)
    return s + u * s * (1 - s)


def exact(case, seed):
    c = case
    v = _inputs(c, seed)
    back = c["kind"].endswith("bwd")
    out = {}
    if c["kind"] == "linear_fwd":
        a = torch.einsum("rk,nk->rn", v["x"].double(), v["W"].double()) + v["bias"].double()
        if c["pre"]:
            out["pre"] = a
    elif c["kind"] == "linear_bwd":
        a = torch.einsum("rn,nk->rk", v["g"].double(), v["W"].double())
        out["dW"] = torch.einsum("rn,rk->nk", v["g"].double(), v["x"].double())
        out["dbias"] = torch.einsum("rn->n", v["g"].double())
    else:
        a = (v["g"] if back else v["x"]).double()
    if not back:
        a = _act_exact(c, a)
    elif v["pre"] is not None:
        a = a * _slope_exact(c, v["pre"].double())
    if c["p"]:
        a = (a * _scale(c)).masked_fill(~_kept_exact(c, v["rng"], *a.shape), 0.0)
    if v["res"] is not None:
        a = a + v["res"].double()
    out["dx" if c["kind"] == "linear_bwd" else "y"] = a
    return out
