"""fp32 rows of the smallest values, and weights that bring them back.  On tensor cores an operand's three bf16 parts
end at bf16's smallest step, 2^-133: beside what other values are off by, a value is off by half of it."""
import numpy as np
import pytest
import torch

import _linear as t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R, K, N", [(74, 256, 256), (2072, 256, 256), (2072, 257, 260)])
def test_small_rows(lib, R, K, N):
    rng = np.random.default_rng(9)
    scale = 2.0 ** -(90 + np.arange(R) % 37.0)  # a row's own, 2^-126 the least
    x = (rng.standard_normal((R, K)) * scale[:, None]).astype(np.float32)
    W = (rng.standard_normal((N, K)) * 2.0 ** 96).astype(np.float32)
    s = lib.make_linear(R, K, N, torch.float32)
    path = lib.linear_path_for_shape(s)
    assert path == (R > 100)
    y = torch.empty(R, N, device="cuda")
    lib.fs_linear_fwd(s, torch.from_numpy(x).cuda(), torch.from_numpy(W).cuda(), None, 0, 0.0, None, None, y, None, lib.linear_workspace(s))
    x, W = x.astype(np.float64), W.astype(np.float64)
    bound = t.sum_bound(K, np.abs(x) @ np.abs(W).T, "f32") + (2.0 ** -134 * np.abs(W).sum(1) if path else 0)
    off = np.abs(t.host(y) - x @ W.T)
    for e in (90, 100, 110, 118, 126):
        i = np.arange(R)[np.arange(R) % 37 == e - 90]
        print(path, e, (off[i] / np.abs(x @ W.T)[i].mean()).max(), (off[i] / bound[i]).max())
    assert (off <= bound).all()
