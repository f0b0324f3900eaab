"""The attention coupling (slice -> q, k, v -> norms -> attention -> deslice) and the layer around it on
the GPU, against the fp64 oracle; tolerances as for the other couplings (tests/_parity.py)."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc

from _parity import error, host, to_dev, tol

pytestmark = pytest.mark.gpu

CASES = [  # B, N, H, d, G, dtype, cap, qk_norm, bias, documents, prefix
    (1, 700, 2, 32, 40, "f32", 0.0, False, False, 0, False),
    (2, 513, 2, 16, 33, "f32", 5.0, True, True, 0, False),
    (1, 900, 1, 64, 64, "f32", 0.0, True, False, 2, False),
    (2, 1500, 2, 32, 130, "f32", 8.0, True, True, 2, True),
    (1, 3000, 2, 32, 64, "bf16", 0.0, True, False, 0, False),
    (2, 2100, 2, 32, 160, "bf16", 10.0, True, False, 3, False),
]


def make(seed, B, N, H, d, G, dtype, cap, qk_norm, bias, docs, prefix):
    rng = np.random.default_rng(seed)

    def n(*s, f=1.0):
        return (f * rng.standard_normal(s)).astype(np.float32)

    def point(x):  # the values that the dtype holds
        return host(to_dev(x, dtype)).astype(np.float32)

    a = {"x_mid": point(n(B, N, H, d)), "fx": point(n(B, N, H, d)), "W_slice": n(H, d, G, f=d ** -0.5),
         "bias": n(H, G, f=0.1), "tau": (0.4 + 0.4 * rng.random(H)).astype(np.float32),
         "Wq": n(H, d, d, f=2 * d ** -0.5), "Wk": n(H, d, d, f=2 * d ** -0.5), "Wv": n(H, d, d, f=d ** -0.5)}
    dout = point(n(B, N, H, d))
    gammas = {"gamma_q": 1 + n(d, f=0.2), "gamma_k": 1 + n(d, f=0.2)} if qk_norm else {}
    mask = {}
    if bias:
        mask["slopes"] = (0.1 * rng.random(H)).astype(np.float32)
    if docs:
        mask["doc_q"] = rng.integers(-1, docs, (B, G)).astype(np.int32)
        mask["doc_k"] = mask["doc_q"].copy()
    if prefix:
        mask["prefix"] = rng.integers(0, G, B).astype(np.int32)
    return a, dout, gammas, mask


def dev(a, dtype):
    return {k: to_dev(v, dtype if k in ("x_mid", "fx") else "f32") for k, v in a.items()}


def device_mask(lib, mask):
    return lib.attn_mask(**{k: torch.from_numpy(v).cuda() for k, v in mask.items()})


@pytest.mark.parametrize("case", CASES, ids=lambda c: "B{}N{}H{}d{}G{}-{}".format(*c[:6]))
def test_forward_and_backward(lib, case):
    B, N, H, d, G, dtype, cap, qk_norm, _, _, prefix = case
    a, dout, gammas, mask = make(sum(case[:5]), *case)
    t, g, m = dev(a, dtype), {k: to_dev(v, "f32") for k, v in gammas.items()}, device_mask(lib, mask)
    c = lib.AttentionCoupling(B, N, H, d, G, torch.bfloat16 if dtype == "bf16" else torch.float32, backward=True, cap=cap,
                              prefix=prefix, qk_norm=qk_norm)
    out = c.forward(**t, mask=m, **g)
    grads = c.backward(**t, dout=to_dev(dout, dtype), mask=m, **g)
    assert c.device_status() == lib.FS_OK
    ref = orc.attention_coupling(**a, **gammas, scale=d ** -0.5, cap=cap, qk_norm=qk_norm, dout=dout, **mask)
    for n, got in {"out": out, **grads}.items():
        e = error(host(got), ref[n], dtype)
        print(f"PARITY attention coupling {case[:6]} {n} {e:.3e}")
        assert e <= tol(dtype), f"{n}: {e:.3e}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_from_the_checkpoint(lib, dtype):
    """The gradients are, bit for bit, those of a coupling that is given the restored inputs; the
    forward's are those of the inputs themselves; two layers share the restored buffers."""
    case = (2, 1000, 2, 32, 64, dtype, 6.0, True, True, 0, False)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    layers, shared = [], None
    for seed in (1, 2):
        a, dout, gammas, mask = make(seed, *case)
        t, g = dev(a, dtype), {k: to_dev(v, "f32") for k, v in gammas.items()}
        c = lib.AttentionCoupling(*case[:5], dt, backward=True, cap=6.0, qk_norm=True, checkpointed=True, restored=shared)
        shared = c.restored
        plain = lib.AttentionCoupling(*case[:5], dt, backward=True, cap=6.0, qk_norm=True)
        m = device_mask(lib, mask)
        assert torch.equal(c.forward(**t, mask=m, **g), plain.forward(**t, mask=m, **g))
        layers.append((a, t, g, m, to_dev(dout, dtype), c, plain))
    for a, t, g, m, do, c, plain in reversed(layers):
        rows = {k: orc.unpack(*orc.pack(a[k].reshape(2000, 64))).reshape(a[k].shape) for k in ("x_mid", "fx")}
        r = {**t, **dev(rows, dtype)}
        plain.forward(**r, mask=m, **g)
        want = plain.backward(**r, dout=do, mask=m, **g)
        weights = {k: v for k, v in t.items() if k not in ("x_mid", "fx")}
        got = c.backward(None, None, **weights, dout=do, mask=m, **g)
        assert c.device_status() == lib.FS_OK
        assert all(torch.equal(got[n], want[n]) for n in want)
        with pytest.raises(ValueError):
            c.backward(**t, dout=do, mask=m, **g)


def test_a_layer_of_norm_projections_and_coupling(lib):
    """norm(stream + update) -> projections -> attention coupling, and back to the stream's gradient
    and the norm's weights, from the stream's 8-bit checkpoint; fp32, against the fp64 chain."""
    B, N, H, d, G = 1, 600, 2, 32, 48
    C, rng = H * d, np.random.default_rng(5)
    n = lambda *s, f=1.0: (f * rng.standard_normal(s)).astype(np.float32)  # noqa: E731
    stream, update, dstream, dout = n(B * N, C, f=2.0), n(B * N, C), n(B * N, C), n(B, N, H, d)
    gamma, beta, Px, Pf = 1 + n(C, f=0.1), n(C, f=0.1), n(C, C, f=C ** -0.5), n(C, C, f=C ** -0.5)
    a, _, _, _ = make(9, B, N, H, d, G, "f32", 0.0, False, False, 0, False)
    weights = {k: v for k, v in a.items() if k not in ("x_mid", "fx")}
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    w = {k: cu(v) for k, v in weights.items()}
    x, r = cu(stream), lib.make_rows(B * N, C)
    y, mean, rstd, (q8, e8) = torch.empty_like(x), torch.empty(B * N, device="cuda"), torch.empty(B * N, device="cuda"), lib.checkpoint(r)
    lib.fs_norm_fwd(r, x, cu(update), cu(gamma), cu(beta), 1e-5, x, y, mean, rstd, q8, e8)
    c = lib.AttentionCoupling(B, N, H, d, G, torch.float32, backward=True)
    xm, fx = ((y.double() @ cu(P).double()).float().view(B, N, H, d) for P in (Px, Pf))
    out = c.forward(xm, fx, **w)
    g = c.backward(xm, fx, **w, dout=cu(dout))
    dy = sum(g[k].view(-1, C).double() @ cu(P).double().T for k, P in (("dx_mid", Px), ("dfx", Pf))).float()
    dgamma, dbeta, ds = torch.empty(C, device="cuda"), torch.empty(C, device="cuda"), cu(dstream)
    lib.fs_norm_bwd(r, None, q8, e8, cu(gamma), mean, rstd, dy, ds, ds, dgamma, dbeta, False, lib.norm_workspace(r))
    v = stream.astype(np.float64) + update
    yr, mr, rr = orc.norm(v, gamma, beta)
    xr, fr = (yr @ P.astype(np.float64) for P in (Px, Pf))
    ref = orc.attention_coupling(xr.reshape(B, N, H, d), fr.reshape(B, N, H, d), **weights, scale=d ** -0.5, dout=dout)
    dyr = ref["dx_mid"].reshape(-1, C) @ Px.astype(np.float64).T + ref["dfx"].reshape(-1, C) @ Pf.astype(np.float64).T
    kept = orc.unpack(*orc.pack((stream + update).astype(np.float32)))
    dvr, dgr, dbr = orc.norm_bwd(kept, gamma, mr, rr, dyr, dstream)
    for name, got, want in (("sum", x, v), ("y", y, yr), ("out", out, ref["out"]), ("dx_mid", g["dx_mid"], ref["dx_mid"]),
                            ("dWq", g["dWq"], ref["dWq"]), ("dv", ds, dvr), ("dgamma", dgamma, dgr), ("dbeta", dbeta, dbr)):
        e = error(host(got).reshape(want.shape), want, "f32")
        print(f"PARITY layer {name} {e:.3e}")
        assert e <= tol("f32"), f"{name}: {e:.3e}"


@pytest.mark.parametrize("case", [(2, 900, 2, 32, 60, "bf16", 6.0, True, True, 2, False), (1, 1200, 8, 32, 500, "f32", 0.0, True, False, 0, True)],
                         ids=["warps", "tcgen05"])
def test_captured_steps_and_two_layers_at_once(lib, case):
    """A step replayed from a graph on new inputs, and two layers' steps on two streams, have the
    bits of steps that run alone."""
    B, N, H, d, G, dtype, cap, _, _, _, prefix = case
    dt, names = torch.bfloat16 if dtype == "bf16" else torch.float32, ("x_mid", "fx")

    def layer(seed):
        a, dout, gammas, mask = make(seed, *case)
        t, g, m, do = dev(a, dtype), {k: to_dev(v, "f32") for k, v in gammas.items()}, device_mask(lib, mask), to_dev(dout, dtype)
        c = lib.AttentionCoupling(*case[:5], dt, backward=True, cap=cap, prefix=prefix, qk_norm=True, checkpointed=True)
        w = {k: v for k, v in t.items() if k not in names}

        def step(stream=None):
            c.forward(**t, mask=m, **g, stream=stream)
            return c.backward(None, None, **w, dout=do, mask=m, **g, stream=stream)

        def result():
            assert c.device_status() == lib.FS_OK
            return {"out": c.out.clone(), **{k: v.clone() for k, v in grads.items()}}

        grads = step()
        return t, step, result, result()

    first, second = layer(1), layer(2)
    t, step, result, alone = first
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in names:
        t[n].copy_(second[0][n])
    graph.replay()
    replayed = result()
    step()
    again = result()
    assert all(torch.equal(replayed[n], again[n]) for n in again) and not torch.equal(again["out"], alone["out"])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for (_, go, _, _), s in zip((first, second), streams):
            go(s)
    torch.cuda.synchronize()
    both = result()
    assert all(torch.equal(both[n], again[n]) for n in again)
    both = second[2]()
    assert all(torch.equal(both[n], second[3][n]) for n in both)


def test_one_token_per_head(lib):
    """G = 1: each point's weight and each attention weight is 1; the scores have no gradient."""
    case = (2, 300, 2, 32, 1, "f32", 0.0, False, False, 0, False)
    a, dout, _, _ = make(3, *case)
    t = dev(a, "f32")
    c = lib.AttentionCoupling(*case[:5], torch.float32, backward=True)
    out = c.forward(**t)
    g = c.backward(**t, dout=to_dev(dout, "f32"))
    ref = orc.attention_coupling(**a, scale=32 ** -0.5, dout=dout)
    for n, got in (("out", out), ("dfx", g["dfx"]), ("dWv", g["dWv"])):
        assert error(host(got), ref[n], "f32") <= tol("f32"), n
    # p (dout . v - dout . out) with out = v: what is left of two equal dot products of 32 terms
    size = np.abs(host(c.d_tokens_mixed) * host(c.tokens_mixed)).sum(-1).max()
    assert np.abs(host(c.dq)).max() <= 32 * 2.0 ** -22 * size * 32 ** -0.5 * np.abs(host(c.k)).max()
