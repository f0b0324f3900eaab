"""Pin of the oracle's attention coupling (CPU): gradients against differences."""
import numpy as np

from oracle import operators_oracle as orc


def test_gradients_are_those_of_differences():
    rng = np.random.default_rng(0)
    B, N, H, d, G = 1, 5, 2, 3, 4
    a = {"x_mid": rng.standard_normal((B, N, H, d)), "fx": rng.standard_normal((B, N, H, d)),
         "W_slice": rng.standard_normal((H, d, G)), "bias": rng.standard_normal((H, G)), "tau": 0.5 + rng.random(H),
         "Wq": rng.standard_normal((H, d, d)), "Wk": rng.standard_normal((H, d, d)), "Wv": rng.standard_normal((H, d, d)),
         "gamma_q": rng.standard_normal(d), "gamma_k": rng.standard_normal(d)}
    dout = rng.standard_normal((B, N, H, d))
    args = dict(scale=0.7, cap=2.0, qk_norm=True, slopes=np.array([0.1, 0.2]), prefix=np.array([2]))
    g = orc.attention_coupling(**a, dout=dout, **args)
    for name in a:
        grad = g["dW" if name == "W_slice" else "d" + name]
        step = rng.standard_normal(a[name].shape)
        f = [(orc.attention_coupling(**{**a, name: a[name] + s * 1e-6 * step}, **args)["out"] * dout).sum() for s in (1, -1)]
        assert abs((f[0] - f[1]) / 2e-6 - (grad * step).sum()) < 1e-6 * max(1.0, abs(grad * step).sum()), name
