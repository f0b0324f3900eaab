"""The linear maps and dropout as a layer uses them: the feed-forward half, and a whole layer (norm,
projections, coupling, projection back with dropout and residual, norm, feed-forward), forward and
backward, against autograd in 64 bits with the oracle's masks; and a captured training step that
draws anew.

Bounds, normwise (largest error by largest value).  fp32: the coupling's outputs and gradients are
within 1e-4 of themselves (its own bar), the other calls within 1e-5; a layer passes an error on through four
products and two norms, which gain less than 10 together on these inputs: 1e-3.  bf16 feed-forward: five
roundings of 2^-8 on the way (hidden rows, gradients, results), and a rounded operand's errors add up
at most: 5 * 2^-8."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc

pytestmark = pytest.mark.gpu

F64 = dict(dtype=torch.float64)


def off(got, want):
    want = want.detach().double().cpu()
    return float((got.double().cpu() - want).abs().max() / want.abs().max())


def mask(R, C, p, rng):
    """What the dropout with these words multiplies by."""
    if not p:
        return 1.0
    seed, step = rng.tolist()
    return torch.tensor(orc.kept(R, C, p, seed, step) / (1 - float(np.float32(p))))


ACTS = {1: torch.relu, 2: torch.nn.functional.gelu, 3: torch.nn.functional.silu}


def feed_forward(x, W1, b1, W2, b2, act, m1, m2):
    return (ACTS[act](x @ W1.T + b1) * m1 @ W2.T + b2) * m2


def parameters(rng, shapes, dtype):
    """Weights in the rows' type, biases in fp32, and the same as leaves in 64 bits."""
    own = [torch.tensor(rng.standard_normal(s) / np.sqrt(s[-1]), dtype=dtype if len(s) == 2 else torch.float32) for s in shapes]
    return [t.cuda() for t in own], [t.double().requires_grad_() for t in own]


@pytest.mark.parametrize("R, C, hidden, act, p", [(1, 32, 64, 2, 0.1), (77, 40, 72, 3, 0.25), (1500, 64, 256, 2, 0.1), (1030, 66, 130, 1, 0.0),
                                                  (3000, 128, 512, 2, 0.1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_feed_forward(lib, dtype, R, C, hidden, act, p):
    rng = np.random.default_rng(R)
    x, res, dy, dres = (torch.tensor(rng.standard_normal((R, C)), dtype=dtype) for _ in range(4))
    own, leaves = parameters(rng, [(hidden, C), (hidden,), (C, hidden), (C,)], dtype)
    words = [lib.dropout_rng(5, i) if p else None for i in range(2)]
    ff = lib.FeedForward(R, C, hidden, dtype, act, p, backward=True)
    xc = x.cuda()
    y = ff.forward(xc, *own, res.cuda(), *words)
    grads = ff.backward(own[0], own[2], dy.cuda(), dres.cuda(), *words)
    masks = [mask(R, c, p, w) for c, w in zip((hidden, C), words)]
    t = x.double().requires_grad_()
    want = feed_forward(t, *leaves, act, *masks) + res.double()
    ((want * dy.double()).sum() + (t * dres.double()).sum()).backward()
    bound = 2e-5 if dtype is torch.float32 else 5 * 2.0 ** -8
    assert off(y, want) < bound
    for name, leaf in zip(("dx", "dW1", "db1", "dW2", "db2"), (t, *leaves)):
        assert off(grads[name], leaf.grad) < bound, name


def test_feed_forward_for_inference_keeps_nothing(lib):
    ff = lib.FeedForward(4, 16, 32)
    assert ff.pre is None and not hasattr(ff, "dW1")


@pytest.mark.parametrize("p", [0.0, 0.1])
def test_layer(lib, p):
    rng = np.random.default_rng(11)
    N, H, d, G, hidden = 1100, 2, 32, 24, 192
    C, dt = H * d, torch.float32
    stream = torch.tensor(rng.standard_normal((N, C)), dtype=dt)
    dout = torch.tensor(rng.standard_normal((N, C)), dtype=dt)
    own, leaves = parameters(rng, [(C, C), (C,), (C, C), (C,), (C, C), (C,), (hidden, C), (hidden,), (C, hidden), (C,)], dt)
    Wx, bx, Wf, bf, Wo, bo, W1, b1, W2, b2 = own
    W = torch.tensor(rng.standard_normal((H, d, G)) / np.sqrt(d), dtype=dt)
    M = torch.tensor(np.eye(G) + 0.1 * rng.standard_normal((H, G, G)), dtype=dt)
    bias, tau = torch.zeros(H, G), torch.full((H,), 0.7)
    words = [lib.dropout_rng(9, i) if p else None for i in range(3)]

    # the library
    rows = lib.make_rows(N, C, dt)
    f32 = dict(device="cuda")
    s0, n1, xm, fx, s1, n2 = (torch.empty(N, C, **f32) for _ in range(6))
    s0.copy_(stream)
    stats = [torch.empty(N, **f32) for _ in range(4)]
    lin = lib.make_linear(N, C, C, dt)
    wf, wb = lib.linear_workspace(lin), lib.linear_workspace(lin, True)
    cp = lib.Coupling(1, N, H, d, G, dt, backward=True)
    ff = lib.FeedForward(N, C, hidden, dt, lib.FS_ACT_GELU, p, backward=True)
    cu = [v.cuda() for v in (W, bias, tau, M)]
    lib.fs_norm_fwd(rows, s0, None, None, None, 1e-5, None, n1, stats[0], stats[1])
    lib.fs_linear_fwd(lin, n1, Wx, bx, 0, 0.0, None, None, xm, None, wf)
    lib.fs_linear_fwd(lin, n1, Wf, bf, 0, 0.0, None, None, fx, None, wf)
    mixed = cp.forward(xm, fx, *cu)
    lib.fs_linear_fwd(lin, mixed, Wo, bo, 0, p, words[0], s0, s1, None, wf)
    lib.fs_norm_fwd(rows, s1, None, None, None, 1e-5, None, n2, stats[2], stats[3])
    y = ff.forward(n2, W1, b1, W2, b2, s1, *words[1:])

    dy = dout.cuda()
    ds1, dmixed, dn1, ds0, g = (torch.empty(N, C, **f32) for _ in range(5))
    gr = ff.backward(W1, W2, dy, None, *words[1:])
    lib.fs_norm_bwd(rows, s1, None, None, None, stats[2], stats[3], gr["dx"], dy, ds1, None, None, False, lib.norm_workspace(rows))
    lib.fs_dropout_bwd(rows, ds1, 0, p, words[0], None, g)
    new = lambda: (torch.empty(C, C, **f32), torch.empty(C, **f32))  # noqa: E731
    (dWo, dbo), (dWx, dbx), (dWf, dbf) = new(), new(), new()
    lib.fs_linear_bwd(lin, mixed, Wo, g, 0, 0.0, None, None, None, dmixed, dWo, dbo, False, wb)
    cg = cp.backward(xm, fx, *cu, dmixed)
    lib.fs_linear_bwd(lin, n1, Wx, cg["dx_mid"], 0, 0.0, None, None, None, dn1, dWx, dbx, False, wb)
    lib.fs_linear_bwd(lin, n1, Wf, cg["dfx"], 0, 0.0, None, None, dn1, dn1, dWf, dbf, False, wb)  # both ways join
    lib.fs_norm_bwd(rows, s0, None, None, None, stats[0], stats[1], dn1, ds1, ds0, None, None, False, lib.norm_workspace(rows))
    torch.cuda.synchronize()

    # 64 bits
    t = stream.double().requires_grad_()
    lWx, lbx, lWf, lbf, lWo, lbo, l1, lb1, l2, lb2 = leaves
    Wd, Md = W.double().requires_grad_(), M.double().requires_grad_()

    def norm(v):
        v = v - v.mean(1, keepdim=True)
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5)

    a = norm(t)
    pts = [(a @ w.T + b).view(N, H, d).transpose(0, 1) for w, b in ((lWx, lbx), (lWf, lbf))]
    w = torch.softmax((pts[0] @ Wd + bias.double()[:, None]) / tau.double()[:, None, None], -1)
    z = (w.transpose(1, 2) @ pts[1]) / (w.sum(1)[..., None] + 1e-5)
    back = (w @ (Md @ z)).transpose(0, 1).reshape(N, C)
    one = t + (back @ lWo.T + lbo) * mask(N, C, p, words[0])
    want = one + feed_forward(norm(one), l1, lb1, l2, lb2, 2, mask(N, hidden, p, words[1]), mask(N, C, p, words[2]))
    (want * dout.double()).sum().backward()
    assert off(y, want) < 1e-3
    for got, leaf in ((ds0, t), (dWx, lWx), (dbx, lbx), (dWf, lWf), (dbf, lbf), (dWo, lWo), (dbo, lbo), (gr["dW1"], l1), (gr["db1"], lb1),
                      (gr["dW2"], l2), (gr["db2"], lb2), (cg["dW"], Wd), (cg["dM"], Md)):
        assert off(got, leaf.grad) < 1e-3


def test_a_captured_step_draws_anew(lib):
    """A training step in a graph: the offsets are advanced in device memory between replays."""
    R, C, hidden, p = 700, 64, 128, 0.2
    g = torch.Generator(device="cuda").manual_seed(1)
    x, res, dy = (torch.randn(R, C, generator=g, device="cuda").bfloat16() for _ in range(3))
    W1, W2 = (torch.randn(*s, generator=g, device="cuda").bfloat16() / 8 for s in ((hidden, C), (C, hidden)))
    b1, b2 = torch.zeros(hidden, device="cuda"), torch.zeros(C, device="cuda")
    words = lib.dropout_rng(3, 0), lib.dropout_rng(3, 1)
    ff = lib.FeedForward(R, C, hidden, p=p, backward=True)

    def step():
        ff.forward(x, W1, b1, W2, b2, res, *words)
        ff.backward(W1, W2, dy, res, *words)
        for w in words:
            w[1] += 2

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (ff.y, ff.dx, ff.dW1, ff.db1, ff.dW2, ff.db2)]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    eager = []
    for w, o in zip(words, (0, 1)):
        w[1] = o
    for _ in range(3):
        step()
        eager.append(results())
    for w, o in zip(words, (0, 1)):
        w[1] = o
    for k in range(3):
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), eager[k]))
    assert not torch.equal(eager[0][0], eager[1][0])
