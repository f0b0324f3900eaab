"""Pins of the oracle's layer norm and 8-bit checkpoint (CPU): closed forms, finite differences,
autograd in 64 bits, and the checkpoint's error bound."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc


def test_norm_by_hand():
    y, mean, rstd = orc.norm(np.array([[1.0, 3.0]]), gamma=[2.0, 2.0], beta=[1.0, 0.0], eps=0.0)
    assert mean[0] == 2.0 and rstd[0] == 1.0 and np.array_equal(y, [[-1.0, 2.0]])


def test_norm_gradient_is_that_of_differences():
    rng = np.random.default_rng(0)
    v, dy = rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    ga, be, dres = rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    _, mean, rstd = orc.norm(v, ga, be)
    dv, dg, db = orc.norm_bwd(v, ga, mean, rstd, dy, dres)

    def loss(v, ga, be):
        return (orc.norm(v, ga, be)[0] * dy).sum() + (v * dres).sum()

    h = 1e-6
    for r in range(3):
        for c in range(7):
            e = np.zeros_like(v)
            e[r, c] = h
            assert abs((loss(v + e, ga, be) - loss(v - e, ga, be)) / (2 * h) - dv[r, c]) < 1e-7
    for c in range(7):
        e = np.eye(7)[c] * h
        assert abs((loss(v, ga + e, be) - loss(v, ga - e, be)) / (2 * h) - dg[c]) < 1e-7
        assert abs((loss(v, ga, be + e) - loss(v, ga, be - e)) / (2 * h) - db[c]) < 1e-7


def test_norm_gradient_is_that_of_autograd():
    rng = np.random.default_rng(1)
    v = torch.tensor(rng.standard_normal((5, 33)), requires_grad=True)
    ga = torch.tensor(rng.standard_normal(33), requires_grad=True)
    dy = rng.standard_normal((5, 33))
    torch.nn.functional.layer_norm(v, (33,), ga, None, 1e-5).backward(torch.tensor(dy))
    _, mean, rstd = orc.norm(v.detach().numpy(), ga.detach().numpy())
    dv, dg, _ = orc.norm_bwd(v.detach().numpy(), ga.detach().numpy(), mean, rstd, dy)
    assert np.abs(dv - v.grad.numpy()).max() < 1e-12 and np.abs(dg - ga.grad.numpy()).max() < 1e-12


def test_pack_by_hand():
    # largest magnitude 1: steps of 2^-6; 127.5 steps would round past 127, so 2^-5 there
    q, e = orc.pack(np.array([[1.0, -0.5, 2.0 ** -7, 3 * 2.0 ** -7]]))
    assert e[0, 0] == 127 - 6 and q.tolist() == [[64, -32, 0, 2]]  # ties to even
    q, e = orc.pack(np.array([[127.5 / 64]]))
    assert e[0, 0] == 127 - 5 and q[0, 0] == 64
    q, e = orc.pack(np.array([[np.nextafter(np.float32(127.5 / 64), np.float32(0))]]))
    assert e[0, 0] == 127 - 6 and q[0, 0] == 127
    q, e = orc.pack(np.zeros((1, 3)))
    assert e[0, 0] == 1 and not q.any()
    assert np.isnan(orc.unpack(*orc.pack(np.array([[1.0, np.inf], [np.nan, 0.0]])))).all()


@pytest.mark.parametrize("C", [1, 31, 32, 33, 100])
def test_pack_is_half_a_step_off_at_most(C):
    rng = np.random.default_rng(C)
    x = (rng.standard_normal((20, C)) * np.exp(3 * rng.standard_normal((20, 1)))).astype(np.float32)
    q, e = orc.pack(x)
    off = np.abs(orc.unpack(q, e) - x)
    step = np.repeat(np.ldexp(1.0, e.astype(int) - 127), 32, axis=1)[:, :C]
    assert (off <= step / 2).all()
    assert np.abs(q.astype(int)).max() <= 127
