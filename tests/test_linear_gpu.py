"""Linear maps of rows and dropout on the GPU against the fp64 oracle (bounds: _linear.py)."""
import threading

import numpy as np
import pytest
import torch

import _linear as t
from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu

# rows, Cin, Cout: one of each, odd ones, both sides of tiles of 64, 128 and 256, few rows and many
SIZES = [(1, 1, 1), (1, 7, 5), (1, 1024, 100), (3, 130, 1), (4, 256, 1030), (5, 64, 33), (17, 8, 8), (63, 31, 65), (64, 64, 64),
         (100, 64, 66), (127, 100, 101), (129, 256, 128), (200, 72, 136), (255, 136, 264), (257, 200, 72), (300, 330, 198),
         (513, 96, 320), (1000, 33, 257), (1030, 520, 40), (600, 700, 72), (3000, 601, 131), (2051, 64, 264), (70, 2049, 130), (30000, 24, 40), (4100, 520, 1032), (9000, 328, 600),
         (20000, 256, 256), (3000, 1100, 72), (4100, 518, 1030),
         (1300, 301, 555), (40, 8192, 300), (40, 300, 8192), (70000, 256, 1),
         (70000, 3, 100), (140000, 320, 3), (140000, 4, 240)]


@pytest.mark.parametrize("R, K, N", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(lib, dtype, R, K, N):
    t.check_forward(lib, R, K, N, dtype, seed=R)
    t.check_forward(lib, R, K, N, dtype, "gelu", 0.25, res=True, pre=True, seed=R + 1)
    t.check_forward(lib, R, K, N, dtype, "silu", 0.0, bias=False, pre=True, seed=R + 2)
    t.check_forward(lib, R, K, N, dtype, "relu", 0.1, res=True, inplace=True, seed=R + 3)


@pytest.mark.parametrize("R, K, N", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(lib, dtype, R, K, N):
    t.check_backward(lib, R, K, N, dtype, seed=R)
    t.check_backward(lib, R, K, N, dtype, "gelu", 0.25, dres=True, accumulate=True, seed=R + 1)
    t.check_backward(lib, R, K, N, dtype, "silu", 0.0, dres=True, inplace=True, want_db=False, seed=R + 2)
    t.check_backward(lib, R, K, N, dtype, "relu", 0.1, want_dw=False, seed=R + 3)
    t.check_backward(lib, R, K, N, dtype, want_dx=False, accumulate=True, seed=R + 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R, K, N", [(5, 40, 24), (700, 264, 328), (700, 331, 263), (1700, 264, 328), (1700, 331, 263)])
def test_non_finite_values_stay_where_they_enter(lib, dtype, R, K, N):
    rng = np.random.default_rng(5)
    x, W, g = (t.tensor(rng, s, dtype) for s in ((R, K), (N, K), (R, N)))
    s = lib.make_linear(R, K, N, t.DTYPES[dtype])
    y, dx = torch.empty(R, N, dtype=x.dtype, device="cuda"), torch.empty_like(x)
    dW, db = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    wf, wb = lib.linear_workspace(s), lib.linear_workspace(s, True)
    x[R - 1, K - 1], x[2, 3] = float("nan"), float("inf")
    g[R - 2, N - 1], g[1, 2] = float("inf"), float("nan")
    lib.fs_linear_fwd(s, x, W, None, 2, 0.0, None, None, y, None, wf)
    lib.fs_linear_bwd(s, x, W, g, 0, 0.0, None, None, None, dx, dW, db, False, wb)
    bad = torch.zeros(R, dtype=torch.bool, device="cuda")
    bad[[R - 1, 2]] = True
    assert torch.isfinite(y[~bad]).all() and torch.isnan(y[R - 1]).all()
    # gelu: an infinity, or 0 where it is negative
    assert not (torch.isfinite(y[2]) & (y[2] != 0)).any()
    bad.zero_()
    bad[[R - 2, 1]] = True
    assert torch.isfinite(dx[~bad]).all() and not torch.isfinite(dx[bad]).any()
    # dW[n, k] sums g[:, n] x[:, k]
    hit = torch.zeros(N, K, dtype=torch.bool, device="cuda")
    hit[[N - 1, 2]] = True
    hit[:, [K - 1, 3]] = True
    assert torch.isfinite(dW[~hit]).all() and not torch.isfinite(dW[hit]).any()
    assert torch.isfinite(db[[i for i in range(N) if i not in (2, N - 1)]]).all()
    assert torch.isnan(db[2]) and torch.isinf(db[N - 1])
    # W: one row makes one channel non-finite
    W[N // 2, 0] = float("nan")
    lib.fs_linear_fwd(s, g.new_zeros(R, K).add_(1), W, None, 0, 0.0, None, None, y, None, wf)
    ok = torch.arange(N, device="cuda") != N // 2
    assert torch.isfinite(y[:, ok]).all() and torch.isnan(y[:, ~ok]).all()


@pytest.mark.parametrize("R", [64, 2048])
def test_fp32_values_up_to_the_largest(lib, R):
    """Rows of fp32's largest values and weights that bring them back: nothing on the way is infinite."""
    rng = np.random.default_rng(6)
    K = N = 256
    top = np.float32(np.finfo(np.float32).max)
    x = (top * rng.uniform(0.97, 1.0, (R, K)).astype(np.float32) * rng.choice(np.float32([-1, 1]), (R, K))).astype(np.float32)
    x[:, 0] = top
    W = (rng.standard_normal((N, K)) * 2.0 ** -30).astype(np.float32)
    s = lib.make_linear(R, K, N, torch.float32)
    assert lib.linear_path_for_shape(s) == (R == 2048)
    y = torch.empty(R, N, device="cuda")
    lib.fs_linear_fwd(s, torch.from_numpy(x).cuda(), torch.from_numpy(W).cuda(), None, 0, 0.0, None, None, y, None, lib.linear_workspace(s))
    x, W = x.astype(np.float64), W.astype(np.float64)
    assert (np.abs(t.host(y) - x @ W.T) <= t.sum_bound(K, np.abs(x) @ np.abs(W).T, "f32")).all()


WIDTHS = [1, 2, 3, 4, 5, 6, 8, 12, 30, 31, 32, 64, 66, 100, 198, 255, 256, 1000, 8192]


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropout(lib, dtype, C):
    rng = np.random.default_rng(C)
    for R, act, p, with_res in ((1, "none", 0.5, False), (7, "gelu", 0.1, True), (133, "silu", 0.25, True), (70, "relu", 0.0, False),
                                (2003 if C < 300 else 40, "gelu", 0.9, True)):
        x, res = t.tensor(rng, (R, C), dtype, 2.0), t.tensor(rng, (R, C), dtype)
        rows, rnd = lib.rows_of(x), lib.dropout_rng(t.SEED, t.STEP) if p else None
        y, tail = t.spare((R, C), x.dtype)
        lib.fs_dropout_fwd(rows, x, t.ACTS.index(act), p, rnd, res if with_res else None, y)
        a = orc.activation(act, t.host(x))[0]
        want = orc.dropout(a, p, t.SEED, t.STEP) + (t.host(res) if with_res else 0)
        off = t.act_off(a, t.host(x), dtype) if act in ("gelu", "silu") else 0
        bound = (off + 3 * t.U * np.abs(a)) / (1 - p) + (2 * t.U + 1.01 * t.HALF[dtype]) * np.abs(want) + 1e-30
        bound = bound + (2 * t.U * np.abs(t.host(res)) if with_res else 0)
        assert (np.abs(t.host(y) - want) <= bound).all() and t.untouched(tail)
        if not with_res and p:
            assert np.array_equal(t.host(y) != 0, orc.kept(R, C, p, t.SEED, t.STEP) & (a != 0))
        dx, tail = t.spare((R, C), x.dtype)
        lib.fs_dropout_bwd(rows, res, t.ACTS.index(act), p, rnd, x if act != "none" else None, dx)
        slope = orc.activation(act, t.host(x))[1]
        want = orc.dropout(t.host(res) * slope, p, t.SEED, t.STEP)
        off = {"none": 0.0, "relu": 0.0}.get(act, 32 * t.U if dtype == "f32" else 1.2e-4)
        bound = off * np.abs(t.host(res)) / (1 - p) + (4 * t.U + 1.01 * t.HALF[dtype]) * np.abs(want) + 1e-30
        assert (np.abs(t.host(dx) - want) <= bound).all() and t.untouched(tail)
        # in place: over x, over the residual, over the gradient, over the pre-activations
        for over in ("x", "res"):
            bufs = {"x": x.clone(), "res": res.clone()}
            lib.fs_dropout_fwd(rows, bufs["x"], t.ACTS.index(act), p, rnd, bufs["res"] if with_res else None, bufs[over])
            assert torch.equal(bufs[over], y) or over == "res" and not with_res
            lib.fs_dropout_bwd(rows, bufs["res"].copy_(res), t.ACTS.index(act), p, rnd, bufs["x"].copy_(x), bufs[over])
            assert torch.equal(bufs[over], dx)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_activations_everywhere(lib, dtype, act):
    """Dense over the whole range, and the special values."""
    u = np.concatenate([np.linspace(-130, 130, 40001), np.linspace(-6, 6, 40001), 10.0 ** np.arange(-38, 38),
                        -10.0 ** np.arange(-38, 38)]).astype(np.float32)
    x = torch.from_numpy(u).cuda().to(t.DTYPES[dtype])[None]
    y, dx = torch.empty_like(x), torch.empty_like(x)
    a, s = orc.activation(act, t.host(x))
    lib.fs_dropout_fwd(lib.rows_of(x.view(-1, 1)), x, t.ACTS.index(act), 0.0, None, None, y)
    lib.fs_dropout_bwd(lib.rows_of(x.view(-1, 1)), torch.ones_like(x), t.ACTS.index(act), 0.0, None, x, dx)
    tiny = 2.0 ** -126
    if dtype == "f32":
        # Phi(-a): quotients 2 u each, the polynomial with its argument 4, the exponential 4 (2 units in the last
        # place), four products; the sigmoid: exponential 4, reciprocal 2, two products
        assert (np.abs(t.host(y) - a) <= 16 * t.U * np.abs(a) + tiny).all()
        assert (np.abs(t.host(dx) - s) <= 32 * t.U + tiny).all()
    else:
        assert (np.abs(t.host(y) - a) <= (2.0 ** -12 + 1.01 * 2.0 ** -8) * np.abs(a) + 2e-7).all()
        assert (np.abs(t.host(dx) - s) <= 1.2e-4 + 1.01 * 2.0 ** -8 * np.abs(s)).all()
    z = torch.tensor([[float("inf"), float("-inf"), float("nan"), 0.0, -0.0]], device="cuda", dtype=x.dtype)
    y, dx, rows = torch.empty_like(z), torch.empty_like(z), lib.rows_of(z)
    lib.fs_dropout_fwd(rows, z, t.ACTS.index(act), 0.0, None, None, y)
    lib.fs_dropout_bwd(rows, torch.ones_like(z), t.ACTS.index(act), 0.0, None, z, dx)
    y, dx = y[0].tolist(), dx[0].tolist()
    assert y[0] == float("inf") and y[1] == 0 and y[2] != y[2] and y[3] == 0 and y[4] == 0
    assert dx[0] == 1 and dx[1] == 0 and dx[2] != dx[2]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dropped_values_are_not_looked_at(lib, dtype):
    R, C, p = 50, 36, 0.5
    keep = torch.from_numpy(orc.kept(R, C, p, t.SEED, t.STEP)).cuda()
    x = torch.full((R, C), float("nan"), device="cuda", dtype=t.DTYPES[dtype])
    x[keep] = 1.0
    y = torch.empty_like(x)
    lib.fs_dropout_fwd(lib.rows_of(x), x, lib.FS_ACT_NONE, p, lib.dropout_rng(t.SEED, t.STEP), None, y)
    assert torch.equal(y, torch.where(keep, 2.0, 0.0).to(x.dtype))


def test_the_product_and_the_dropout_call_draw_the_same_mask(lib):
    for R, K, N, dtype in ((1, 64, 40, "bf16"), (300, 256, 264, "bf16"), (257, 40, 101, "bf16"), (300, 64, 70, "f32")):
        rng = np.random.default_rng(0)
        x, W = t.tensor(rng, (R, K), dtype), t.tensor(rng, (N, K), dtype)
        s, rnd = lib.make_linear(R, K, N, x.dtype), lib.dropout_rng(4, 5)
        y, z = (torch.empty(R, N, dtype=x.dtype, device="cuda") for _ in range(2))
        ws = lib.linear_workspace(s)
        lib.fs_linear_fwd(s, x, W, None, 0, 0.25, rnd, None, y, None, ws)
        lib.fs_dropout_fwd(lib.rows_of(z), torch.ones_like(z), 0, 0.25, rnd, None, z)
        assert torch.equal(y != 0, z != 0)


@pytest.mark.parametrize("R, K, N, dtype", [(9, 40, 24, "bf16"), (3000, 256, 264, "bf16"), (3000, 100, 66, "f32"), (3000, 300, 200, "f32"), (3000, 201, 301, "f32"),
                                           (700, 33, 65, "bf16"), (700, 333, 165, "bf16")])
def test_calls_repeat_to_the_bit_and_graphs_draw_anew(lib, R, K, N, dtype):
    rng = np.random.default_rng(1)
    x, W, g, pre = (t.tensor(rng, s, dtype) for s in ((R, K), (N, K), (R, N), (R, K)))
    s, rnd = lib.make_linear(R, K, N, x.dtype), lib.dropout_rng(4, 5)
    out = {n: torch.empty(z, dtype=d, device="cuda") for n, z, d in
           (("y", (R, N), x.dtype), ("dx", (R, K), x.dtype), ("dW", (N, K), torch.float32), ("db", (N,), torch.float32))}
    wf, wb = lib.linear_workspace(s), lib.linear_workspace(s, True)

    def step():
        lib.fs_linear_fwd(s, x, W, None, 2, 0.3, rnd, None, out["y"], None, wf)
        lib.fs_linear_bwd(s, x, W, g, 2, 0.3, rnd, pre, None, out["dx"], out["dW"], out["db"], False, wb)

    def now():
        torch.cuda.synchronize()
        return {n: v.clone() for n, v in out.items()}

    step()
    first = now()
    step()
    assert all(torch.equal(v, first[n]) for n, v in now().items())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(v, first[n]) for n, v in now().items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for v in out.values():
        v.fill_(7)
    graph.replay()
    assert all(torch.equal(v, first[n]) for n, v in now().items())
    rnd[1] += 1
    graph.replay()
    other = now()
    assert not torch.equal(other["y"], first["y"]) and not torch.equal(other["dx"], first["dx"])
    assert torch.equal(other["dW"], first["dW"])
    step()
    assert all(torch.equal(v, other[n]) for n, v in now().items())


def test_calls_of_two_host_threads(lib):
    rng = np.random.default_rng(2)
    jobs, errors = [], []
    for R, K, N, dtype in ((500, 256, 136, "bf16"), (500, 40, 72, "f32")):
        x, W = t.tensor(rng, (R, K), dtype), t.tensor(rng, (N, K), dtype)
        s = lib.make_linear(R, K, N, x.dtype)
        y, ws = torch.empty(R, N, dtype=x.dtype, device="cuda"), lib.linear_workspace(s)
        lib.fs_linear_fwd(s, x, W, None, 0, 0.0, None, None, y, None, ws)
        jobs.append((s, x, W, y.clone(), y, ws))
    torch.cuda.synchronize()

    def run(s, x, W, want, y, ws):
        try:
            stream = torch.cuda.Stream()
            for _ in range(30):
                with torch.cuda.stream(stream):
                    y.fill_(7)
                    lib.fs_linear_fwd(s, x, W, None, 0, 0.0, None, None, y, None, ws)
                stream.synchronize()
                assert torch.equal(y, want)
        except BaseException as e:  # noqa: BLE001  (handed to the test's thread)
            errors.append(e)

    threads = [threading.Thread(target=run, args=j) for j in jobs]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not errors, errors


def test_a_workspace_of_another_shape_before(lib):
    """What a workspace holds does not matter."""
    rng = np.random.default_rng(3)
    R, K, N = 400, 264, 200
    x, W = t.tensor(rng, (R, K), "bf16"), t.tensor(rng, (N, K), "bf16")
    s = lib.make_linear(R, K, N, x.dtype)
    ys = []
    for fill in (0, 255):
        ws = torch.full((lib.linear_workspace_bytes(s),), fill, dtype=torch.uint8, device="cuda")
        y = torch.empty(R, N, dtype=x.dtype, device="cuda")
        lib.fs_linear_fwd(s, x, W, None, 0, 0.0, None, None, y, None, ws)
        ys.append(y)
    assert torch.equal(*ys)
