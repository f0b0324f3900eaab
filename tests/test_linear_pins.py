"""Pins of the oracle's linear maps, activations and dropout (CPU): the generator's published
test vectors, closed forms, autograd in 64 bits and differences."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc

ACTS = {"none": lambda u: u, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}


@pytest.mark.parametrize("counter, key, want", [
    # the generator's authors' known answers
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator(counter, key, want):
    assert tuple(int(w) for w in orc.philox(np.array(counter), key)) == want


def test_kept_by_hand():
    # four channels share a counter, a row begins a new one
    k = orc.kept(3, 6, 0.5, 7 + (5 << 32), 9 + (11 << 32))
    for r in range(3):
        for c in range(6):
            w = orc.philox(np.array([2 * r + c // 4, 0, 9, 11]), (7, 5))[c % 4]
            assert k[r, c] == (w >= 1 << 31)
    assert orc.kept(4, 5, 2.0 ** -40, 1, 2).all()


@pytest.mark.parametrize("p", [0.1, 0.25, 0.9])
def test_kept_share(p):
    # 400,000 draws: five standard deviations
    n = 400000
    share = orc.kept(1000, 400, p, 3, 4).mean()
    assert abs(share - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n)


@pytest.mark.parametrize("act", list(ACTS))
def test_activations(act):
    u = torch.linspace(-9, 9, 181, dtype=torch.float64)[1::2].requires_grad_()  # 0 left out
    y = ACTS[act](u)
    y.sum().backward()
    a, s = orc.activation(act, u.detach().numpy())
    assert np.abs(a - y.detach().numpy()).max() < 1e-14 and np.abs(s - u.grad.numpy()).max() < 1e-14
    a, s = orc.activation(act, np.array([np.inf, -np.inf, np.nan, 0.0]))
    assert a[0] == np.inf and a[1] == (-np.inf if act == "none" else 0) and np.isnan(a[2]) and a[3] == 0
    if act != "none":
        assert s[0] == 1 and s[1] == 0 and np.isnan(s[2])


@pytest.mark.parametrize("act", list(ACTS))
def test_gradients_are_those_of_autograd_and_of_differences(act):
    """Two maps in a row: the second one's backward goes through the first's activation and dropout."""
    rng = np.random.default_rng(3)
    R, A, B, C = 5, 6, 7, 3
    x, W1, b1 = rng.standard_normal((R, A)), rng.standard_normal((B, A)), rng.standard_normal(B)
    W2, b2, res, dy = (rng.standard_normal(s) for s in ((C, B), (C,), (R, C), (R, C)))

    def forward(x, W1, b1, W2, b2):
        h, u = orc.linear(x, W1, b1, act, 0.25, 12, 13)
        return orc.linear(h, W2, b2, res=res)[0], h, u

    _, h, u = forward(x, W1, b1, W2, b2)
    g, dW2, db2 = orc.linear_bwd(h, W2, dy, act, 0.25, 12, 13, u)
    dx, dW1, db1 = orc.linear_bwd(x, W1, g, dres=2 * x)
    t = [torch.tensor(v, requires_grad=True) for v in (x, W1, b1, W2, b2)]
    keep = torch.tensor(orc.kept(R, B, 0.25, 12, 13))
    hid = ACTS[act](t[0] @ t[1].T + t[2]) * keep / 0.75
    ((hid @ t[3].T + t[4] + torch.tensor(res)) * torch.tensor(dy)).sum().add((t[0] ** 2).sum()).backward()
    for got, leaf in zip((dx, dW1, db1, dW2, db2), t):
        assert np.abs(got - leaf.grad.numpy()).max() < 1e-13
    base = [x, W1, b1, W2, b2]
    for k, got in enumerate((dx - 2 * x, dW1, db1, dW2, db2)):
        for at in np.ndindex(got.shape):
            e = np.zeros_like(base[k])
            e[at] = 1e-6
            up, down = ([v + s * e if i == k else v for i, v in enumerate(base)] for s in (1, -1))
            d = ((forward(*up)[0] - forward(*down)[0]) * dy).sum() / 2e-6
            assert abs(d - got[at]) < 1e-7
