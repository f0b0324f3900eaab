"""dbias of fp32 rows, by the norm of its error.

Bound 3e-7 = 5 u (u = 2^-24).  hi's sums are of values with 8 bits: few of them lose anything at a step.  The
small parts' sums are 2^-8 of hi's, so that their cuts are 2^-8 of a result's step.  What is left are fp32's
roundings, at most u of the running sum each (u / 2 as a rule) and of random sign: a segment's two
halves, up to 14 segments of a part and 7 parts of a chain of the sizes here, and 8 chains: 30 roundings
add up to sqrt(30) u / 2 = 2.8 u of the largest running sum.  One accumulator for all parts is cut 48 times in
256 terms, hi's step each time and always towards zero: 10 u and more."""
import numpy as np
import pytest
import torch

import _linear as t
import _tensor_core as tc

BOUND = 3e-7


def rows(R, N, shift):
    return (np.random.default_rng(21).standard_normal((R, N)) + shift).astype(np.float32)


@pytest.mark.parametrize("R, shift", [(2048, 0.0), (2048, 0.25), (16384, 0.0)])
def test_the_bound_tells_one_accumulator_from_two(R, shift):
    g = rows(R, 256, shift)
    hi, mid, lo = (p.T for p in tc.parts(g))
    ones, want = np.ones((1, R)), g.astype(np.float64).sum(0)
    one = tc.sums([(0, lo, ones), (0, mid, ones), (0, hi, ones)], R, 512)[:, 0]
    two = tc.sums([(1, lo, ones), (1, mid, ones), (0, hi, ones)], R, 512)[:, 0]
    assert tc.off(two, want) < BOUND < tc.off(one, want)
    assert tc.off(hi.sum(1), want) > 1000 * BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N, shift", [(2048, 256, 256, 0.0), (2048, 256, 256, 0.25), (16384, 256, 256, 0.0), (131072, 256, 256, 0.0),
                                            (20001, 201, 250, 0.0), (900, 256, 2048, 0.0), (4000, 300, 300, 0.0), (300, 40, 30, 0.0)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_dbias(lib, R, K, N, shift, accumulate):
    """Out of the product (Cin up to 256), by kernels of its own, and in multiply-adds."""
    g = rows(R, N, shift)
    x = t.tensor(np.random.default_rng(22), (R, K), "f32")
    s = lib.make_linear(R, K, N, torch.float32)
    dW, db = torch.empty(N, K, device="cuda"), torch.zeros(N, device="cuda")
    if accumulate:
        dW.zero_()
    lib.fs_linear_bwd(s, x, None, torch.from_numpy(g).cuda(), 0, 0.0, None, None, None, None, dW, db, accumulate,
                      lib.linear_workspace(s, True))
    off = tc.off(t.host(db), g.astype(np.float64).sum(0))
    print(R, K, N, accumulate, off)
    assert off < BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N", [(1 << 20, 300, 64), (1 << 20, 258, 65), (300001, 2048, 40)])
def test_dbias_of_many_rows(lib, R, K, N):
    """By kernels of their own (Cin above 256): 128 sums of eight rows in turn, 3 additions in pairs, 8 threads, 16 parts and
    3 additions of the chains are about 160 roundings by u / 2 at most, of running sums whose squares are half of the
    result's on average: sqrt(160 / 2) u / 2 = 4.5 u."""
    gen = torch.Generator(device="cuda").manual_seed(23)
    x, g = (torch.randn(s, generator=gen, device="cuda") for s in ((R, K), (R, N)))
    s = lib.make_linear(R, K, N, torch.float32)
    dW, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    lib.fs_linear_bwd(s, x, None, g, 0, 0.0, None, None, None, None, dW, db, False, lib.linear_workspace(s, True))
    off = tc.off(t.host(db), t.host(g.double().sum(0)))
    print(R, K, N, off)
    assert off < BOUND
