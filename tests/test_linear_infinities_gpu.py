"""Infinities in fp32 maps: results are finite, infinite or NaN as sums in 64 bits are, on both paths.  Weights
of few bits among them, whose smaller bf16 parts are 0."""
import numpy as np
import pytest
import torch

import _linear as t

pytestmark = pytest.mark.gpu
INF = float("inf")


def kind(a):
    """0 finite, 1 and -1 infinities, 2 NaN."""
    return np.where(np.isnan(a), 2.0, np.where(np.isinf(a), np.sign(a), 0.0))


def product(a, b):
    with np.errstate(invalid="ignore"):
        return a @ b


@pytest.mark.parametrize("R, K, N", [(64, 256, 256), (7, 256, 64), (2048, 256, 256), (2051, 263, 255), (2050, 258, 262)])
def test_infinities(lib, R, K, N):
    rng = np.random.default_rng(8)
    x, W, g = (rng.standard_normal(s).astype(np.float32) for s in ((R, K), (N, K), (R, N)))
    W[: N // 2] = rng.choice(np.float32([1, -1, 0.5, -2, 1.25]), (N // 2, K))
    W[1, 0] = 0
    x[3, 0], x[5, K - 1], x[R - 1, 1], x[R - 1, 2], x[6, 0], x[6, 1] = INF, -INF, INF, -INF, INF, INF
    g[2, 0], g[4, N - 1], g[0, 1], g[0, 2] = -INF, INF, INF, INF
    s = lib.make_linear(R, K, N, torch.float32)
    xd, Wd, gd = (torch.from_numpy(a).cuda() for a in (x, W, g))
    y, dx = torch.empty(R, N, device="cuda"), torch.empty(R, K, device="cuda")
    dW, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    lib.fs_linear_fwd(s, xd, Wd, None, 0, 0.0, None, None, y, None, lib.linear_workspace(s))
    lib.fs_linear_bwd(s, xd, Wd, gd, 0, 0.0, None, None, None, dx, dW, db, False, lib.linear_workspace(s, True))
    x, W, g = (a.astype(np.float64) for a in (x, W, g))
    for got, want in ((y, product(x, W.T)), (dx, product(g, W)), (dW, product(g.T, x)), (db, g.sum(0))):
        assert np.array_equal(kind(t.host(got)), kind(want)) and not np.isfinite(want).all()
    # in W, and where both operands have one
    W[2, 1], W[N - 1, K - 1] = INF, -INF
    lib.fs_linear_fwd(s, xd, torch.from_numpy(W).float().cuda(), None, 0, 0.0, None, None, y, None, lib.linear_workspace(s))
    assert np.array_equal(kind(t.host(y)), kind(product(x, W.T)))


@pytest.mark.parametrize("R", [64, 2048])
def test_a_residual_takes_an_infinity_on(lib, R):
    x, W, res = torch.ones(R, 256, device="cuda"), torch.full((256, 256), 0.5, device="cuda"), torch.zeros(R, 256, device="cuda")
    x[1, 1], res[1, 3], x[2, 5] = INF, -INF, -INF
    s = lib.make_linear(R, 256, 256, torch.float32)
    y = torch.empty_like(res)
    lib.fs_linear_fwd(s, x, W, None, lib.FS_ACT_RELU, 0.0, None, res, y, None, lib.linear_workspace(s))
    assert torch.isnan(y[1, 3]) and (y[1, 4:] == INF).all() and (y[2] == 0).all() and (y[3:] == 128).all()
