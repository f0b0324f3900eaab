"""Layer norm and 8-bit checkpoints on the GPU against the fp64 oracle.

Tolerances, elementwise, with u = 2^-24 (fp32's half step) and t the output type's half step
(bf16 2^-8, fp32 2^-24).  A row's sum goes through at most 16 additions in a thread, 5 in a
warp and 16 over warps, so with the products and the division by C a row's average is off by
at most 40 u of the average magnitude.  The mean enters the centred values, these the variance
(two roundings more each, and half of its relative error in rstd)."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
WIDTHS = [1, 2, 3, 4, 16, 30, 31, 32, 64, 65, 66, 100, 101, 196, 198, 255, 256, 257, 300, 384, 512, 513, 1000, 1023, 1024, 1026, 2048, 2050, 4095, 4100,
          5001, 8192]


def tensor(rng, shape, dtype, scale=1.0, shift=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale + shift).astype(np.float32)).to("cuda", DTYPES[dtype])


def host(t):
    return t.double().cpu().numpy()


def spare(shape, dtype, extra=64):
    """An output inside a longer buffer: nothing behind it may be written."""
    n = int(np.prod(shape))
    fill = 7 if dtype in (torch.int8, torch.uint8) else 7.0
    buf = torch.full((n + extra,), fill, dtype=dtype, device="cuda")
    return buf[:n].view(shape), buf[n:]


def untouched(*tails):
    return all(bool((t == 7).all()) for t in tails)


def norm_bounds(v, gamma, beta, rstd, mean, y, dtype):
    a, d = np.abs(v).mean(1, keepdims=True), np.abs(v - mean[:, None])
    g = 1.0 if gamma is None else np.abs(gamma)
    b = 0.0 if beta is None else np.abs(beta)
    r = rstd[:, None]
    # the squared centred values' error in rstd: twice the mean's error against the deviation
    return (g * r * (40 * U * a + 40 * U * d) + g * r * r * d * 80 * U * a + 4 * U * (np.abs(y) + b)
            + HALF[dtype] * 1.01 * np.abs(y) + 1e-30)


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(lib, dtype, C):
    rng = np.random.default_rng(C)
    for rows, with_res, with_ckpt in ((1, False, False), (7, True, True), (133, True, False), (70, False, True)):
        x = tensor(rng, (rows, C), dtype, 2.0, 0.5)
        res = tensor(rng, (rows, C), dtype) if with_res else None
        gamma, beta = tensor(rng, (C,), "f32"), tensor(rng, (C,), "f32")
        r = lib.rows_of(x)
        y, t0 = spare((rows, C), DTYPES[dtype])
        s, t1 = spare((rows, C), DTYPES[dtype])
        mean, t2 = spare((rows,), torch.float32)
        rstd, t3 = spare((rows,), torch.float32)
        q8, t4 = spare((rows, C), torch.int8)
        e8, t5 = spare((rows, (C + 31) // 32), torch.uint8)
        lib.fs_norm_fwd(r, x, res, gamma, beta, 1e-5, s if with_res else None, y, mean, rstd,
                        q8 if with_ckpt else None, e8 if with_ckpt else None)
        torch.cuda.synchronize()
        assert untouched(t0, t1, t2, t3, t4, t5)
        v = host(x)
        if with_res:
            kept = (x.float() + res.float()).to(DTYPES[dtype])
            assert torch.equal(s, kept)
            v = host(kept)
        else:
            assert untouched(s.flatten())
        want, m, rs = orc.norm(v, host(gamma), host(beta))
        assert (np.abs(host(mean) - m) <= 41 * U * np.abs(v).mean(1)).all()
        far = 45 * U * rs + rs * rs * 41 * U * np.abs(v).mean(1)
        assert (np.abs(host(rstd) - rs) <= far).all()
        assert (np.abs(host(y) - want) <= norm_bounds(v, host(gamma), host(beta), rs, m, want, dtype)).all()
        if with_ckpt:
            q, e = orc.pack(v)
            assert np.array_equal(q8.cpu().numpy(), q) and np.array_equal(e8.cpu().numpy(), e)
        else:
            assert untouched(q8.flatten(), e8.flatten())


def backward_bounds(v, gamma, mean, rstd, dy, dv, dtype, terms):
    xh = (v - mean[:, None]) * rstd[:, None]
    g = dy if gamma is None else dy * gamma
    avg1, avg2 = np.abs(g).mean(1, keepdims=True), np.abs(g * xh).mean(1, keepdims=True)
    r = rstd[:, None]
    tol = r * (42 * U * avg1 + np.abs(xh) * 48 * U * avg2 + 6 * U * (np.abs(g) + avg1 + np.abs(xh) * avg2))
    # (v - mean) rstd: two roundings; the difference is exact to u of itself
    tol = tol + 4 * U * np.abs(dv) + HALF[dtype] * 1.01 * np.abs(dv) + 1e-30
    return tol, (terms + 4) * U * np.abs(dy * xh).sum(0) + 1e-30, terms * U * np.abs(dy).sum(0) + 1e-30


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(lib, dtype, C):
    rng = np.random.default_rng(5000 + C)
    for rows, with_res, with_ckpt, accumulate in ((1, False, False, False), (7, True, True, False),
                                                  (133, True, False, True), (70, False, True, True)):
        v = tensor(rng, (rows, C), dtype, 2.0, 0.5)
        dy = tensor(rng, (rows, C), dtype)
        dres = tensor(rng, (rows, C), dtype) if with_res else None
        gamma = tensor(rng, (C,), "f32")
        r = lib.rows_of(v)
        q8 = e8 = None
        vh = host(v)
        if with_ckpt:
            q8, e8 = lib.checkpoint(r)
            lib.fs_ckpt_pack(r, v, q8, e8)
            vh = orc.unpack(*orc.pack(vh))
        _, m, rs = orc.norm(host(v))
        mean, rstd = torch.tensor(m, dtype=torch.float32, device="cuda"), torch.tensor(rs, dtype=torch.float32, device="cuda")
        dv, t0 = spare((rows, C), DTYPES[dtype])
        dgamma, t1 = spare((C,), torch.float32)
        dbeta, t2 = spare((C,), torch.float32)
        old_g, old_b = host(dgamma), host(dbeta)
        ws = lib.norm_workspace(r)
        lib.fs_norm_bwd(r, None if with_ckpt else v, q8, e8, gamma, mean, rstd, dy, dres, dv, dgamma, dbeta, accumulate,
                        ws)
        assert lib.fs_device_status(ws) == lib.FS_OK
        assert untouched(t0, t1, t2)
        want, dg, db = orc.norm_bwd(vh, host(gamma), host(mean), host(rstd), host(dy),
                                    host(dres) if with_res else None)
        # a column's sum: at most rows + 64 additions in whatever order
        tol, tg, tb = backward_bounds(vh, host(gamma), host(mean), host(rstd), host(dy), want, dtype, rows + 64)
        assert (np.abs(host(dv) - want) <= tol).all()
        if accumulate:
            dg, db = dg + old_g, db + old_b
        assert (np.abs(host(dgamma) - dg) <= tg + 2 * U * np.abs(dg)).all()
        assert (np.abs(host(dbeta) - db) <= tb + 2 * U * np.abs(db)).all()


@pytest.mark.parametrize("C", [32, 100, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(lib, dtype, C):
    """More rows than one round of the blocks takes: every row, and the whole column sums."""
    rng = np.random.default_rng(C)
    rows = 70001
    v, dy = tensor(rng, (rows, C), dtype), tensor(rng, (rows, C), dtype)
    r = lib.rows_of(v)
    y, mean, rstd = torch.empty_like(v), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    q8, e8 = lib.checkpoint(r)
    lib.fs_norm_fwd(r, v, None, None, None, 1e-5, None, y, mean, rstd, q8, e8)
    back = torch.empty_like(v)
    lib.fs_ckpt_unpack(r, q8, e8, back)
    dv, dg, db = torch.empty_like(v), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    lib.fs_norm_bwd(r, v, None, None, None, mean, rstd, dy, None, dv, dg, db, False, lib.norm_workspace(r))
    vh = host(v)
    want, m, rs = orc.norm(vh)
    assert (np.abs(host(y) - want) <= norm_bounds(vh, None, None, rs, m, want, dtype)).all()
    at = rng.integers(0, rows, 200)
    assert np.array_equal(host(back)[at], orc.unpack(*orc.pack(vh[at])))
    wv, wg, wb = orc.norm_bwd(vh, None, host(mean), host(rstd), host(dy))
    # a thread adds at most rows / 152 values of a column in turn, then 8 warps, 19 + 32 partial sums
    tol, tg, tb = backward_bounds(vh, None, host(mean), host(rstd), host(dy), wv, dtype, rows / 152 + 64)
    assert (np.abs(host(dv) - wv) <= tol).all()
    assert (np.abs(host(dg) - wg) <= tg).all() and (np.abs(host(db) - wb) <= tb).all()


@pytest.mark.parametrize("rows", [15, 16, 17, 70_001])
@pytest.mark.parametrize("C, dtype", [(65, "bf16"), (101, "f32"), (255, "bf16"), (255, "f32")])
def test_forward_of_odd_rows_in_stages(lib, rows, C, dtype):
    """Rows that come by bulk copies, 16 at a time: the stream in place of either input, its checkpoint,
    the norm; the formula in 64 bits on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(rows + C)
    new = lambda *n: torch.randn(*n, generator=g, device="cuda").to(DTYPES[dtype])  # noqa: E731
    x, res, gamma, beta = new(rows, C), new(rows, C), new(C).float(), new(C).float()
    r = lib.rows_of(x)
    v = (x.float() + res.float()).to(DTYPES[dtype])
    want8, want_e = lib.checkpoint(r)
    lib.fs_ckpt_pack(r, v, want8, want_e)

    def forward(x, res, to):
        y, t0 = spare((rows, C), DTYPES[dtype])
        mean, t1 = spare((rows,), torch.float32)
        rstd, t2 = spare((rows,), torch.float32)
        q8, t3 = spare((rows, C), torch.int8)
        e8, t4 = spare(tuple(want_e.shape), torch.uint8)
        lib.fs_norm_fwd(r, x, res, gamma, beta, 1e-5, to, y, mean, rstd, q8, e8)
        torch.cuda.synchronize()
        assert untouched(t0, t1, t2, t3, t4)
        return to, y, mean, rstd, q8, e8

    got = forward(x, res, torch.empty_like(x))
    s, y, mean, rstd, q8, e8 = got
    assert torch.equal(s, v) and torch.equal(q8, want8) and torch.equal(e8, want_e)
    d = v.double()
    m = d.mean(1)
    rs = torch.rsqrt(d.var(1, unbiased=False) + 1e-5)
    want = (d - m[:, None]) * rs[:, None] * gamma.double() + beta.double()
    a = d.abs().mean(1)
    assert bool(((mean - m).abs() <= 41 * U * a).all())
    assert bool(((rstd - rs).abs() <= 45 * U * rs + rs * rs * 41 * U * a).all())
    # as in norm_bounds
    far, g, k = (d - m[:, None]).abs(), gamma.double().abs(), rs[:, None]
    tol = (g * k * (40 * U * a[:, None] + 40 * U * far) + g * k * k * far * 80 * U * a[:, None]
           + 4 * U * (want.abs() + beta.double().abs()) + HALF[dtype] * 1.01 * want.abs() + 1e-30)
    assert bool(((y.double() - want).abs() <= tol).all())
    for inputs in ((x.clone(), res), (x, res.clone())):
        to = inputs[0] if inputs[0] is not x else inputs[1]
        assert all(torch.equal(p, q) for p, q in zip(forward(*inputs, to), got))


@pytest.mark.parametrize("rows, C, dtype", [(240_011, 256, "bf16"), (233_472, 256, "bf16"), (70_001, 512, "bf16"), (70_001, 384, "bf16"),
                                            (70_001, 300, "bf16"), (70_001, 101, "bf16"), (70_001, 101, "f32"),
                                            (70_001, 420, "f32"), (15, 512, "bf16"), (16, 512, "bf16"), (17, 101, "bf16"),
                                            (30_000, 255, "f32"), (30_000, 511, "bf16")])
@pytest.mark.parametrize("with_res, with_ckpt", [(False, False), (True, True), (True, False), (False, True)])
def test_backward_of_rows_in_stages(lib, rows, C, dtype, with_res, with_ckpt):
    """Rows that come by bulk copies, 16 at a time: whole stages, a last one of fewer rows, several rounds of the
    stages; out of place, and in place of either gradient.  The formula in 64 bits on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(rows + C)
    new = lambda *n: torch.randn(*n, generator=g, device="cuda").to(DTYPES[dtype])  # noqa: E731
    v, dy, dres, gamma = new(rows, C), new(rows, C), new(rows, C) if with_res else None, new(C).float()
    r = lib.rows_of(v)
    mean, rstd = v.float().mean(1), torch.rsqrt(v.float().var(1, unbiased=False) + 1e-5)
    q8 = e8 = None
    x = v.double()
    if with_ckpt:
        q8, e8 = lib.checkpoint(r)
        lib.fs_ckpt_pack(r, v, q8, e8)
        scale = torch.exp2(e8.double() - 127).repeat_interleave(32, 1)[:, :C]
        x = q8.double() * scale
    ws = lib.norm_workspace(r)

    def backward(dy, dres, to):
        dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        lib.fs_norm_bwd(r, None if with_ckpt else v, q8, e8, gamma, mean, rstd, dy, dres, to, dg, db, False, ws)
        assert lib.fs_device_status(ws) == lib.FS_OK
        return to, dg, db

    buf, tail = spare((rows, C), DTYPES[dtype])
    dv, dg, db = backward(dy, dres, buf)
    assert untouched(tail)
    y, m, rs = dy.double(), mean.double()[:, None], rstd.double()[:, None]
    xh = (x - m) * rs
    gg = y * gamma.double()
    a1, a2 = gg.abs().mean(1, keepdim=True), (gg * xh).abs().mean(1, keepdim=True)
    want = rs * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True))
    if with_res:
        want = want + dres.double()
    # as in backward_bounds
    tol = rs * (42 * U * a1 + xh.abs() * 48 * U * a2 + 6 * U * (gg.abs() + a1 + xh.abs() * a2))
    tol = tol + 4 * U * want.abs() + HALF[dtype] * 1.01 * want.abs() + 1e-30
    if with_res:
        tol = tol + 2 * U * dres.double().abs()
    assert bool(((dv.double() - want).abs() <= tol).all())
    terms = min(rows, rows / 152 + 64) + 64
    assert bool(((dg.double() - (y * xh).sum(0)).abs() <= (terms + 4) * U * (y * xh).abs().sum(0) + 1e-30).all())
    assert bool(((db.double() - y.sum(0)).abs() <= terms * U * y.abs().sum(0) + 1e-30).all())
    a = dy.clone()
    assert all(torch.equal(p, q) for p, q in zip(backward(a, dres, a), (dv, dg, db)))
    if with_res:
        b = dres.clone()
        assert all(torch.equal(p, q) for p, q in zip(backward(dy, b, b), (dv, dg, db)))


@pytest.mark.parametrize("C", [1, 5, 31, 32, 33, 62, 64, 200, 256, 1030, 8192])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_checkpoint_is_exact(lib, dtype, C):
    rng = np.random.default_rng(C)
    rows = 37
    x = rng.standard_normal((rows, C)) * np.exp(4 * rng.standard_normal((rows, 1)))
    x[0] = 0.0
    x[1] = 2.0 ** -130                      # below the smallest step
    x[2] = 3.3e38
    x[3] = 127.5 / 64                       # rounds past 127 at the smaller step
    x[4] = np.nextafter(np.float32(127.5 / 64), np.float32(0))
    x[5] = (np.arange(C) % 128 + 0.5) / 64  # ties
    x[6, C // 2] = np.nan
    x[7, 0] = np.inf
    x[8, -1] = -np.inf
    x[9] = -0.0
    x[10] = 2.0 ** -126
    t = torch.from_numpy(x.astype(np.float32)).to("cuda", DTYPES[dtype])
    r = lib.rows_of(t)
    q8, t0 = spare((rows, C), torch.int8)
    e8, t1 = spare((rows, (C + 31) // 32), torch.uint8)
    back, t2 = spare((rows, C), DTYPES[dtype])
    lib.fs_ckpt_pack(r, t, q8, e8)
    lib.fs_ckpt_unpack(r, q8, e8, back)
    torch.cuda.synchronize()
    assert untouched(t0, t1, t2)
    q, e = orc.pack(host(t))
    assert np.array_equal(e8.cpu().numpy(), e) and np.array_equal(q8.cpu().numpy(), q)
    assert np.array_equal(host(back), orc.unpack(q, e), equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(lib, dtype):
    """The stream's sum over x or res, and dv over dy or dres, give what separate buffers give."""
    rng = np.random.default_rng(3)
    rows, C = 301, 256
    x, res, dy = (tensor(rng, (rows, C), dtype) for _ in range(3))
    r = lib.rows_of(x)
    f32 = dict(device="cuda")

    def forward(x, res, s):
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, **f32), torch.empty(rows, **f32)
        lib.fs_norm_fwd(r, x, res, None, None, 1e-5, s, y, mean, rstd)
        return s, y, mean, rstd

    want = forward(x, res, torch.empty_like(x))
    a, b = x.clone(), res.clone()
    for got in (forward(a, res, a), forward(x, b, b)):
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    s, _, mean, rstd = want
    ws = lib.norm_workspace(r)

    def backward(dy, dres, dv):
        lib.fs_norm_bwd(r, s, None, None, None, mean, rstd, dy, dres, dv, None, None, False, ws)
        return dv

    dv = backward(dy, res, torch.empty_like(x))
    a, b = dy.clone(), res.clone()
    assert torch.equal(backward(a, res, a), dv) and torch.equal(backward(dy, b, b), dv)


def test_from_the_checkpoint_as_from_its_values(lib):
    """fp32 rows hold the checkpoint's values exactly: the same bits either way."""
    rng = np.random.default_rng(4)
    v, dy = tensor(rng, (500, 96), "f32"), tensor(rng, (500, 96), "f32")
    r = lib.rows_of(v)
    q8, e8 = lib.checkpoint(r)
    mean, rstd = v.mean(1), 1 / v.std(1)
    lib.fs_ckpt_pack(r, v, q8, e8)
    lib.fs_ckpt_unpack(r, q8, e8, v)
    got = []
    for args in ((v, None, None), (None, q8, e8)):
        dv, dg, db = torch.empty_like(v), torch.empty(96, device="cuda"), torch.empty(96, device="cuda")
        lib.fs_norm_bwd(r, *args, None, mean, rstd, dy, None, dv, dg, db, False, lib.norm_workspace(r))
        got.append((dv, dg, db))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_mean_far_larger_than_the_deviation(lib):
    rng = np.random.default_rng(5)
    x = tensor(rng, (64, 256), "f32", 1.0, 1000.0)
    r = lib.rows_of(x)
    y, mean, rstd = torch.empty_like(x), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    lib.fs_norm_fwd(r, x, None, None, None, 1e-5, None, y, mean, rstd)
    want, m, rs = orc.norm(host(x))
    # the mean's error shifts every value; it enters the variance squared only
    assert (np.abs(host(y) - want) <= norm_bounds(host(x), None, None, rs, m, want, "f32")).all()


def test_constant_rows_and_rows_with_nan(lib):
    x = torch.full((6, 100), 3.0, device="cuda")
    x[2, 7] = float("nan")
    x[4, 99] = float("inf")
    beta = torch.arange(100, dtype=torch.float32, device="cuda")
    r = lib.rows_of(x)
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    lib.fs_norm_fwd(r, x, None, None, beta, 1e-5, None, y, mean, rstd)
    for i in range(6):
        if i in (2, 4):
            assert not torch.isfinite(y[i]).any()
        else:
            # (3 - mean) is at most 40 u times 3, times rstd <= 1 / sqrt(eps)
            assert bool(((y[i] - beta).abs() <= 40 * U * 3 * 320 + U * beta).all())


def test_another_stream_a_graph_and_repeated_runs(lib):
    rng = np.random.default_rng(6)
    rows, C = 3001, 256
    x, dy = tensor(rng, (rows, C), "bf16"), tensor(rng, (rows, C), "bf16")
    r = lib.rows_of(x)
    ws, ckpt = lib.norm_workspace(r), lib.checkpoint(r)
    o = {k: torch.empty_like(x) for k in ("y", "dv")}
    p = {k: torch.empty(n, device="cuda") for k, n in (("mean", rows), ("rstd", rows), ("dg", C), ("db", C))}

    def step(stream=None):
        lib.fs_norm_fwd(r, x, None, None, None, 1e-5, None, o["y"], p["mean"], p["rstd"], *ckpt, stream=stream)
        lib.fs_norm_bwd(r, None, *ckpt, None, p["mean"], p["rstd"], dy, None, o["dv"], p["dg"], p["db"], False, ws,
                        stream=stream)

    step()
    want = [t.clone() for t in (*o.values(), *p.values())]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (*o.values(), *p.values())))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in (*o.values(), *p.values()):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (*o.values(), *p.values())))
