"""Linear maps and dropout of tensors past 2^31 and 2^32 values, against 64 bits at rows on both
sides of these borders and at the last ones (bounds: _linear.py)."""
import numpy as np
import pytest
import torch

import _linear as t
from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu


def rows_at(R, C):
    at = {0, 1, R - 1, R - 2, R // 2}
    for border in (1 << 31, 1 << 32):
        at |= {r for r in (border // C - 1, border // C, border // C + 1) if r < R}
    return sorted(at)


def filled(R, C, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(R, C, generator=g, device="cuda", dtype=dtype)


def dropped(a, at, C, p, seed, offset):
    """orc.dropout of rows `at` of a long tensor."""
    out = np.empty_like(a)
    quads = -(-C // 4)
    for i, r in enumerate(at):
        n = np.arange(r * quads, (r + 1) * quads, dtype=np.uint64)
        c = np.empty((quads, 4), np.uint64)
        c[:, 0], c[:, 1], c[:, 2], c[:, 3] = n & np.uint64(0xFFFFFFFF), n >> np.uint64(32), offset & 0xFFFFFFFF, offset >> 32
        w = orc.philox(c, (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1)[:C]
        out[i] = np.where(w >= int(float(np.float32(p)) * 2.0 ** 32), a[i] / (1 - float(np.float32(p))), 0.0)
    return out


@pytest.mark.parametrize("R, C", [((1 << 32) // 1000 + 700, 1000), ((1 << 32) // 33 + 100, 33)])
def test_dropout(lib, R, C):
    x = filled(R, C, torch.bfloat16, 1)
    y = torch.empty_like(x)
    lib.fs_dropout_fwd(lib.rows_of(x), x, lib.FS_ACT_NONE, 0.25, lib.dropout_rng(t.SEED, t.STEP), None, y)
    at = rows_at(R, C)
    a = t.host(x[at])
    want = dropped(a, at, C, 0.25, t.SEED, t.STEP)
    assert (np.abs(t.host(y[at]) - want) <= (t.HALF["bf16"] * 1.01 + 3 * t.U) * np.abs(want)).all()


@pytest.mark.parametrize("K, N, R, dtype", [(16, 1024, (1 << 32) // 1024 + 300, "bf16"), (1024, 16, (1 << 32) // 1024 + 300, "bf16"),
                                            (40, 1001, (1 << 31) // 1001 + 300, "f32")])
def test_linear(lib, K, N, R, dtype):
    """y, or x, and in the backward g, or dx, past the borders."""
    dt = t.DTYPES[dtype]
    x, W = filled(R, K, dt, 2), filled(N, K, dt, 3)
    s, rnd = lib.make_linear(R, K, N, dt), lib.dropout_rng(t.SEED, t.STEP)
    y = torch.empty(R, N, dtype=dt, device="cuda")
    lib.fs_linear_fwd(s, x, W, None, 0, 0.25, rnd, None, y, None, lib.linear_workspace(s))
    at = rows_at(R, max(K, N))
    u = t.host(x[at]) @ t.host(W).T
    want = dropped(u, at, N, 0.25, t.SEED, t.STEP)
    du = t.sum_bound(K, np.abs(t.host(x[at])) @ np.abs(t.host(W)).T, dtype) + 3 * t.U * np.abs(u)
    assert (np.abs(t.host(y[at]) - want) <= du / 0.75 + 1.01 * t.HALF[dtype] * np.abs(want)).all()
    # backward with y for g
    dx = torch.empty_like(x)
    dW, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    lib.fs_linear_bwd(s, x, W, y, 0, 0.0, None, None, None, dx, dW, db, False, lib.linear_workspace(s, True))
    want = t.host(y[at]) @ t.host(W)
    bound = t.sum_bound(N, np.abs(t.host(y[at])) @ np.abs(t.host(W)), dtype) + 1.01 * t.HALF[dtype] * np.abs(want)
    assert (np.abs(t.host(dx[at]) - want) <= bound).all()
    # the sums over all rows, in 64 bits, a slice of rows at a time
    ww, wb = (torch.zeros(z, dtype=torch.float64, device="cuda") for z in ((N, K), (N,)))
    aw, ab = torch.zeros_like(ww), torch.zeros_like(wb)
    for r in range(0, R, 1 << 18):
        b, a = y[r:r + (1 << 18)].double(), x[r:r + (1 << 18)].double()
        ww += b.T @ a
        aw += b.T.abs() @ a.abs()
        wb += b.sum(0)
        ab += b.abs().sum(0)
    assert ((dW - ww).abs() <= t.sum_bound(R, aw, "f32")).all() and ((db - wb).abs() <= t.sum_bound(R, ab, "f32")).all()
