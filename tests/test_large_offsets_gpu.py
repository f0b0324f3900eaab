"""Calls whose tensors pass 2^31 values: offsets beyond 32 bits.  Rows are independent of one another, so the
results of one call are those of calls on parts of it, bit for bit; the attention's heads are compared with
64 bits.

Of the attention: roundings of either sign stay within 3e-6 of the terms that a result is summed from, and a
weight 2^x with x = s f - lse log2(e) has the roundings of numbers up to |lse| log2(e) (and 24) in its exponent,
of one sign for a row: 4 ln(2) u of them (tests/_attn.py).  lse: 60 u of a product's magnitudes, at most 12
here; at most 1000 tiles added in turn; 140 u for the rest."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def _fill(t, seed):
    """Normal values, made once for the first 2^24 and repeated with a sign and a shift by block."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat, n = t.view(-1), 1 << 24
    base = torch.randn(n, generator=g, device="cuda")
    for i, part in enumerate(flat.split(n)):
        part.copy_(base[:part.numel()].roll(i * 1009) * (1.0 if i % 3 else -1.0))
    return t


# the kernels of the norm: one warp a row by bulk copies or not, eight lanes, a block; a checkpoint each
@pytest.mark.parametrize("C, dtype", [(256, torch.bfloat16), (255, torch.bfloat16), (32, torch.float32), (1024, torch.bfloat16)])
def test_rows(lib, C, dtype):
    rows = (1 << 31) // C + 4099
    new = lambda: torch.empty(rows, C, dtype=dtype, device="cuda")  # noqa: E731
    x, res = _fill(new(), 1), _fill(new(), 2)
    gamma, beta = (torch.randn(C, device="cuda") for _ in range(2))
    r = lib.make_rows(rows, C, dtype)
    parts = [(a, min(rows, a + rows // 3 + 1)) for a in range(0, rows, rows // 3 + 1)]

    def forward(a, b, out):
        s, y, mean, rstd, q8, e8 = out
        lib.fs_norm_fwd(lib.make_rows(b - a, C, dtype), x[a:b], res[a:b], gamma, beta, 1e-5, s, y, mean, rstd, q8, e8)

    def buffers(n):
        f = torch.empty
        return [f(n, C, dtype=dtype, device="cuda"), f(n, C, dtype=dtype, device="cuda"), f(n, device="cuda"),
                f(n, device="cuda"), *lib.checkpoint(lib.make_rows(n, C, dtype))]

    whole = buffers(rows)
    forward(0, rows, whole)
    for a, b in parts:
        # a part starts on a 16-byte boundary
        a -= a % 16
        mine = buffers(b - a)
        forward(a, b, mine)
        assert all(torch.equal(w[a:b], m) for w, m in zip(whole, mine))
        del mine
    s, y, mean, rstd, q8, e8 = whole
    lib.fs_ckpt_pack(r, s, q8.zero_(), e8.zero_())
    lib.fs_ckpt_unpack(r, q8, e8, y)
    for a in (0, (1 << 31) // C - 7, rows - 20):  # around the border and at the ends
        want = q8[a:a + 20].double() * torch.exp2(e8[a:a + 20].double() - 127).repeat_interleave(32, 1)[:, :C]
        assert torch.equal(y[a:a + 20].double(), want)
        step = torch.exp2(e8[a:a + 20].double() - 128).repeat_interleave(32, 1)[:, :C]
        assert bool(((s[a:a + 20].double() - want).abs() <= step).all())

    def backward(a, b, from_ckpt, dv, dg, db, accumulate):
        n = lib.make_rows(b - a, C, dtype)
        src = (None, q8[a:b], e8[a:b]) if from_ckpt else (s[a:b], None, None)
        ws = lib.norm_workspace(n)
        lib.fs_norm_bwd(n, *src, gamma, mean[a:b], rstd[a:b], x[a:b], res[a:b], dv, dg, db, accumulate, ws)
        assert lib.fs_device_status(ws) == lib.FS_OK

    for from_ckpt in (False, True):
        g = [torch.zeros(C, device="cuda") for _ in range(4)]
        backward(0, rows, from_ckpt, y, g[0], g[1], False)
        at = 0
        for _, b in parts:
            b -= 0 if b == rows else b % 16  # 4 bytes a row of the statistics: parts of 16 rows
            dv = torch.empty(b - at, C, dtype=dtype, device="cuda")
            backward(at, b, from_ckpt, dv, g[2], g[3], at > 0)
            assert torch.equal(y[at:b], dv)
            del dv
            at = b
        # sums of the same values in another order: at most rows / 900 additions in turn and 64 more, of
        # values whose mean magnitude is at most that of unit ones (Cauchy), on both sides
        tol = 2 * U * (rows / 900 + 64) * 1.05 * rows
        assert float((g[0] - g[2]).abs().max()) <= tol and float((g[1] - g[3]).abs().max()) <= tol
        assert float(g[1].abs().max()) > 0


def _exact(q, k, v, g, scale):
    """out, lse, score gradients and weights of one head in 64 bits, and the magnitudes that out and they come from."""
    q, k, v, g = (t.double() for t in (q, k, v, g))
    s = scale * (q @ k.T)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    out = p @ v
    D = (g * out).sum(1, keepdim=True)
    return out, lse, p * (g @ v.T - D) * scale, p, p @ v.abs(), p * (g.abs() @ v.abs().T + D.abs()) * scale


def _rel(lse):
    return 3e-6 + 4 * math.log(2) * U * (float(lse.abs().max()) / math.log(2) + 24)


def _near(got, want, terms, rel):
    off = float((got.double() - want).norm())
    assert math.isfinite(off) and off <= rel * float(terms.norm())


LSE = (60 * 12 + 1000 + 140) * U


def _run(lib, s, q, k, v, do):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:-1], device="cuda")
    ws = lib.attn_workspace(s)
    lib.fs_attn_fwd(s, q, k, v, None, out, lse, ws)
    assert lib.fs_device_status(ws) == lib.FS_OK
    del ws
    ws = lib.attn_workspace(s, True)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    lib.fs_attn_bwd(s, q, k, v, None, out, lse, do, dq, dk, dv, ws)
    assert lib.fs_device_status(ws) == lib.FS_OK
    return out, lse, dq, dk, dv


@pytest.mark.parametrize("rows", [1, 130])
def test_attention_over_many_keys(lib, rows):
    """33 heads of 2^20 keys, d = 64: k, v and their gradients of 2.2e9 values; by warps (1 query) and on tcgen05."""
    H, Gk, d = 33, 1 << 20, 64
    s = lib.make_attn_shape(1, H, rows, d, Gk=Gk)
    assert (lib.attn_path_for_shape(s), lib.attn_path_for_shape(s, True)) == ((0, 0) if rows == 1 else (1, 1))
    k, v = (_fill(torch.empty(1, H, Gk, d, device="cuda"), i) for i in (3, 4))
    q, do = (_fill(torch.empty(1, H, rows, d, device="cuda"), i) for i in (5, 6))
    out, lse, dq, dk, dv = _run(lib, s, q, k, v, do)
    for h in (0, 31, 32):
        o, z, ds, p, o_terms, ds_terms = _exact(q[0, h], k[0, h], v[0, h], do[0, h], d ** -0.5)
        rel = _rel(z)
        assert float((lse[0, h].double() - z).abs().max()) <= LSE
        _near(out[0, h], o, o_terms, rel)
        _near(dq[0, h], ds @ k[0, h].double(), ds_terms @ k[0, h].double().abs(), rel)
        _near(dk[0, h], ds.T @ q[0, h].double(), ds_terms.T @ q[0, h].double().abs(), rel)
        _near(dv[0, h], p.T @ do[0, h].double(), p.T @ do[0, h].double().abs(), rel)
        del o, z, ds, p, o_terms, ds_terms


@pytest.mark.parametrize("Gk", [16, 130])
def test_attention_of_many_queries(lib, Gk):
    """33 heads of 2^20 queries, d = 64: q, out, dq of 2.2e9 values against few keys; by warps and on tcgen05."""
    H, Gq, d = 33, 1 << 20, 64
    s = lib.make_attn_shape(1, H, Gq, d, Gk=Gk)
    assert lib.attn_path_for_shape(s) == lib.attn_path_for_shape(s, True) == (0 if Gk == 16 else 1)
    q, do = (_fill(torch.empty(1, H, Gq, d, device="cuda"), i) for i in (5, 6))
    k, v = (_fill(torch.empty(1, H, Gk, d, device="cuda"), i) for i in (3, 4))
    out, lse, dq, dk, dv = _run(lib, s, q, k, v, do)
    for h in (0, 31, 32):
        sums = [torch.zeros(Gk, d, dtype=torch.float64, device="cuda") for _ in range(4)]
        for a in range(0, Gq, 1 << 17):
            at = slice(a, a + (1 << 17))
            o, z, ds, p, o_terms, ds_terms = _exact(q[0, h, at], k[0, h], v[0, h], do[0, h, at], d ** -0.5)
            rel = _rel(z)
            assert float((lse[0, h, at].double() - z).abs().max()) <= LSE
            _near(out[0, h, at], o, o_terms, rel)
            _near(dq[0, h, at], ds @ k[0, h].double(), ds_terms @ k[0, h].double().abs(), rel)
            x, g = q[0, h, at].double(), do[0, h, at].double()
            for t, w in zip(sums, (ds.T @ x, ds_terms.T @ x.abs(), p.T @ g, p.T @ g.abs())):
                t += w
        _near(dk[0, h], sums[0], sums[1], rel)
        _near(dv[0, h], sums[2], sums[3], rel)
