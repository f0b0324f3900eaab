"""fp32 maps by the norm of their error, and weight gradients of wide maps.

An elementwise bound that holds for any signs, (180 + K / 128) u of the terms' magnitudes, is far above what sums of
random signs are off by: a lost part of an operand passes it.  The norm tells.  Bound 1e-6 = 17 u (u = 2^-24):
* a segment of 256 terms is cut 16 times, by half of a last place of the running sum on average (0.72 u of it), always
  towards zero; the running sum after j of 16 steps has sqrt(j / 16) of the segment's norm: 0.72 u * 11.2 = 8 u, which
  stays the share of a sum of segments, whatever their number;
* the additions of up to 64 segments and 8 + 8 parts in fp32 round by u / 2 of a running sum each, of random sign: 4 u;
* what the three parts leave out, three of nine products and 2^-25 of an operand: 1 u; multiply-adds, chains of 128: 3 u.
Without one of the small products of the highest parts it is 80 u (4.9e-6), without both operands' mid parts' 186 u."""
import numpy as np
import pytest
import torch

import _linear as t
import _tensor_core as tc

BOUND = 1e-6


@pytest.mark.parametrize("R, K, N", [(300, 198, 330), (200, 601, 131), (200, 2048, 200)])
def test_the_bound_sees_each_product(R, K, N):
    rng = np.random.default_rng(1)
    x, W = rng.standard_normal((R, K)).astype(np.float32), (rng.standard_normal((N, K)) / np.sqrt(K)).astype(np.float32)
    X, Y, want = tc.parts(x), tc.parts(W), x.astype(np.float64) @ W.astype(np.float64).T
    names = [(0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)]  # parts of x and W, the small products first

    def off(left_out=None):
        return tc.off(tc.sums([(int(n == (0, 0)) ^ 1, X[n[0]], Y[n[1]]) for n in names if n != left_out], K), want)

    assert off() < BOUND
    for n in names:
        assert off(n) > 4 * BOUND, n


def run(lib, R, K, N, dtype, accumulate, seed=0):
    """The outputs of all three products, and what they are in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x, W, g, y = (torch.randn(s, generator=gen, device="cuda").to(t.DTYPES[dtype]) for s in ((R, K), (N, K), (R, N), (R, N)))
    dx, dW, db = torch.empty_like(x), torch.randn(N, K, generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda")
    old = [v.double() if accumulate else torch.zeros((), dtype=torch.float64, device="cuda") for v in (dW, db)]
    s = lib.make_linear(R, K, N, x.dtype)
    lib.fs_linear_fwd(s, x, W, None, 0, 0.0, None, None, y, None, lib.linear_workspace(s))
    ws = lib.linear_workspace(s, True)
    lib.fs_linear_bwd(s, x, W, g, 0, 0.0, None, None, None, dx, dW, db, accumulate, ws)
    assert int(ws[:4].view(torch.int32)[0]) == 0
    xd, Wd, gd = x.double(), W.double(), g.double()
    want = {"y": xd @ Wd.T, "dx": gd @ Wd, "dW": gd.T @ xd + old[0], "dbias": gd.sum(0) + old[1]}
    return {"y": y, "dx": dx, "dW": dW, "dbias": db}, want


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N", [(100, 64, 66), (300, 330, 198), (40, 2048, 2048), (2048, 256, 256), (3000, 601, 131), (4100, 520, 1032),
                                     (9000, 328, 600), (20000, 256, 64), (20000, 255, 66), (131072, 256, 256)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_fp32(lib, R, K, N, accumulate):
    got, want = run(lib, R, K, N, "f32", accumulate)
    for name in got:
        off = float((got[name].double() - want[name]).norm() / want[name].norm())
        print(R, K, N, name, off)
        assert off < BOUND, name


def up(n, to=256):
    return -(-n // to) * to


def workspace(R, K, N, dtype, pairs):
    """Status word, packed operands, parts of dx where its sums are split, parts of dbias; no part of dW."""
    packed = sum(up(rows * up(C, 8) * 2) for rows, C in ((R, N), (N, K), (R, K)) if dtype == "bf16" and C % 8)
    tiles = -(-R // 256) * (-(-K // 128) if dtype == "f32" else -(-K // up(-(-K // -(-K // 256)), 128)))
    per = up(-(-N // max(1, min(pairs // tiles, N // 512))), 64)
    splits = -(-N // per)
    return 256 + packed + (up(splits * R * up(K, 4) * 4) if splits > 1 else 0) + up(N * 128 * 4)


@pytest.mark.gpu
@pytest.mark.parametrize("R, K, N, walks", [(600, 2304, 2304, True), (600, 2305, 2306, True), (70, 2560, 2817, True), (1030, 4100, 2052, True),
                                            (900, 256, 2048, False), (901, 250, 2047, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_dw_out_of_the_product_itself(lib, dtype, R, K, N, walks, accumulate):
    """Sums that are not split: dW is written, or added to, by the product's epilogue, dbias too where dW has up to two tiles of
    columns.  walks: more tiles than pairs of SMs, which each take several."""
    pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
    columns = 128 if dtype == "f32" else 256
    assert (-(-N // 256) * -(-K // columns) > pairs) == walks
    assert lib.linear_workspace_bytes(lib.make_linear(R, K, N, t.DTYPES[dtype]), True) == workspace(R, K, N, dtype, pairs)
    t.check_backward(lib, R, K, N, dtype, accumulate=accumulate, want_dx=False, seed=R)
    got, want = run(lib, R, K, N, dtype, accumulate)
    for name in ("dW", "dbias"):  # fp32 in both types
        assert float((got[name].double() - want[name]).norm() / want[name].norm()) < BOUND, name
