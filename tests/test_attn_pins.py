"""Pins of the oracle's token attention (CPU): closed forms, autograd in 64 bits, differences."""
import numpy as np
import torch

from oracle import operators_oracle as orc


def test_equal_scores_average_the_visible_values():
    v = np.arange(12.0).reshape(1, 1, 4, 3)
    q = k = np.zeros((1, 1, 4, 3))
    out, lse = orc.attention(q, k, v, 1.0)
    assert np.allclose(out, v.mean(2, keepdims=True)) and np.allclose(lse, np.log(4))
    out, lse = orc.attention(q, k, v, 1.0, prefix=[0])
    assert np.allclose(out[0, 0, 1], v[0, 0, :2].mean(0)) and np.allclose(lse[0, 0], np.log([1, 2, 3, 4]))
    out, _ = orc.attention(q, k, v, 1.0, prefix=[2])
    assert np.allclose(out[0, 0, 0], v[0, 0, :2].mean(0))
    doc = np.array([[0, 1, 0, -1]])
    out, lse = orc.attention(q, k, v, 1.0, doc_q=doc, doc_k=doc)
    assert np.allclose(out[0, 0, 2], v[0, 0, [0, 2]].mean(0)) and (out[0, 0, 3] == 0).all() and lse[0, 0, 3] == -np.inf
    # a bias of log 2 per step: weights halve
    out, _ = orc.attention(q, k, v, 1.0, slopes=[np.log(2)])
    w = 0.5 ** np.arange(4)
    assert np.allclose(out[0, 0, 0], (w / w.sum()) @ v[0, 0])
    # one query, the last of four
    out, _ = orc.attention(q[:, :, :1], k, v, 1.0, slopes=[np.log(2)])
    assert np.allclose(out[0, 0, 0], (w[::-1] / w.sum()) @ v[0, 0])


def test_gradients_are_those_of_autograd():
    rng = np.random.default_rng(0)
    B, H, Hkv, G, d = 2, 4, 2, 6, 5
    q, k, v, g = (torch.tensor(rng.standard_normal((B, n, G, d)), requires_grad=True) for n in (H, Hkv, Hkv, H))
    slopes, pos = rng.random(H), 3 * rng.random((B, G))
    doc = rng.integers(-1, 2, (B, G))
    pre = np.array([1, 4])
    s = 0.7 * q @ k.repeat_interleave(2, 1).transpose(-1, -2)
    a = 1.5 * torch.tanh(s / 1.5) - torch.tensor(slopes)[None, :, None, None] * torch.tensor(
        np.abs(pos[:, :, None] - pos[:, None, :]))[:, None]
    ok = np.stack([orc.visible(G, G, doc[b], doc[b], pre[b]) for b in range(B)])[:, None]
    a = a.masked_fill(~torch.tensor(ok), -np.inf)
    out = torch.nan_to_num(torch.softmax(a, -1)) @ v.repeat_interleave(2, 1)
    out.backward(g.detach())
    n = [t.detach().numpy() for t in (q, k, v, g)]
    o, _, dq, dk, dv = orc.attention(*n[:3], 0.7, 1.5, slopes, pos, pos, doc, doc, pre, dout=n[3])
    assert np.abs(o - out.detach().numpy()).max() < 1e-13
    for mine, t in ((dq, q), (dk, k), (dv, v)):
        want = t.grad.numpy()
        fine = np.isfinite(want)  # rows that see nothing have NaN there
        assert np.abs(mine[fine] - want[fine]).max() < 1e-13


def test_gradients_are_those_of_differences():
    rng = np.random.default_rng(1)
    q, k, v, g = (rng.standard_normal((1, 1, 3, 2)) for _ in range(4))
    args = dict(scale=0.5, cap=1.0, slopes=[0.2], prefix=[2])
    grads = dict(zip("qkv", orc.attention(q, k, v, dout=g, **args)[2:]))
    base = {"q": q, "k": k, "v": v}
    for n in "qkv":
        for at in np.ndindex(3, 2):
            e = np.zeros((1, 1, 3, 2))
            e[(0, 0) + at] = 1e-6
            f = [(orc.attention(**{**base, n: base[n] + s * e}, **args)[0] * g).sum() for s in (1, -1)]
            assert abs((f[0] - f[1]) / 2e-6 - grads[n][(0, 0) + at]) < 1e-8
