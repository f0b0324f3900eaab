"""GELU, SILU and their derivatives of bf16 calls over every finite bf16 value: what is rounded is good to
far less than a rounding.

Bound: half a bf16 step at the value in 64 bits, and what fp32 is off before it (u = 2^-24):
* GELU and SILU: e^(-a^2/2) and e^-a take the rounding of their exponents with them: at most 2.25 roundings of
  126 (a = 13.2) times ln 2, 200 u, for GELU, 1.25 roundings of 126 for SILU; quotients and products 10 u,
  GELU's polynomial 2^-19: 2^-16 of the value.  Below 2^-126 the exponential is 0, which is times 13.2 or 87: 2^-119.
* Derivatives: GELU's tail is off by 2^-19 of 1/2, the product with the density by 8 u of 0.25; SILU's 1 - sigmoid by u, times
  an argument of 17, and a few u more: 2^-19."""
import numpy as np
import pytest
import torch

import _linear as t
from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu


def every_value():
    v = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    return v[torch.isfinite(v)].cuda()


def half_step(a):
    """Of bf16 at a."""
    e = np.floor(np.log2(np.maximum(np.abs(a), 2.0 ** -126)))
    return np.ldexp(0.5, (e - 7).astype(int))


def check(got, want, slope):
    off, bound = np.abs(t.host(got) - want), half_step(want) + (2.0 ** -19 if slope else 2.0 ** -16 * np.abs(want) + 2.0 ** -119)
    bad = off > bound
    print(bad.sum(), "of", bad.size)
    assert not bad.any()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_dropout_calls(lib, act):
    u = every_value()
    y, dx, rows = torch.empty_like(u), torch.empty_like(u), lib.make_rows(u.numel(), 1, u.dtype)
    lib.fs_dropout_fwd(rows, u, t.ACTS.index(act), 0.0, None, None, y)
    lib.fs_dropout_bwd(rows, torch.ones_like(u), t.ACTS.index(act), 0.0, None, u, dx)
    a, s = orc.activation(act, t.host(u))
    check(y, a, False)
    check(dx, s, True)


@pytest.mark.parametrize("R", [200, None])
@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_linear_calls(lib, act, R):
    """Rows of one value and zeros, weights of 1 and 0: u is the value itself, on both paths."""
    u = every_value()
    u = u if R is None else u[torch.arange(R, device="cuda") * (u.numel() // R)]
    R, K, N = u.numel(), 8, 64
    x, W, y = torch.zeros(R, K, dtype=u.dtype, device="cuda"), torch.zeros(N, K, dtype=u.dtype, device="cuda"), torch.empty(R, N, dtype=u.dtype, device="cuda")
    x[:, 0], W[:, 0] = u, 1
    s = lib.make_linear(R, K, N, u.dtype)
    assert lib.linear_path_for_shape(s) == (R > 200)
    lib.fs_linear_fwd(s, x, W, None, t.ACTS.index(act), 0.0, None, None, y, None, lib.linear_workspace(s))
    a, slope = orc.activation(act, t.host(u))
    check(y, np.repeat(a[:, None], N, 1), False)
    # dx: g W is 1 in every channel
    s = lib.make_linear(R, N, K, u.dtype)
    g, W, dx = torch.zeros_like(x), torch.zeros(K, N, dtype=u.dtype, device="cuda"), torch.empty_like(y)
    g[:, 0], W[0] = 1, 1
    assert lib.linear_path_for_shape(s, True) == (R > 200)
    lib.fs_linear_bwd(s, None, W, g, t.ACTS.index(act), 0.0, None, u[:, None].expand(R, N).contiguous(), None, dx, None, None, False,
                      lib.linear_workspace(s, True))
    check(dx, np.repeat(slope[:, None], N, 1), True)
