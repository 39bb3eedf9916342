"""The oracle of the gated delta rule against what fixes it: differences of its own forward, the momentum rule's oracle at mu = 0, and the
limits of its gates."""
import numpy as np
import pytest

from oracle import gdr_oracle as gdr
from oracle import mdn_oracle


def inputs(seed, B=2, T=6, H=4, Hk=2, dk=5, dv=3):
    r = np.random.default_rng(seed)
    k = r.normal(size=(B, T, Hk, dk))
    return dict(q=r.normal(size=(B, T, Hk, dk)), k=k / np.linalg.norm(k, axis=-1, keepdims=True), v=r.normal(size=(B, T, H, dv)),
                g=-r.exponential(size=(B, T, H)), beta=r.uniform(size=(B, T, H)), S0=r.normal(size=(B, H, dk, dv)))


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "S0"])
def test_the_adjoint_is_that_of_the_forward(name):
    x = inputs(1)
    r = np.random.default_rng(2)
    dO, dS = r.normal(size=x["v"].shape), r.normal(size=x["S0"].shape)
    b = gdr.backward(**x, dO=dO, dS=dS, scale=0.7)
    def loss(y):
        f = gdr.forward(**y, scale=0.7)
        return (f["o"] * dO).sum() + (f["S"] * dS).sum()
    d, h = r.normal(size=x[name].shape), 1e-5
    num = (loss({**x, name: x[name] + h * d}) - loss({**x, name: x[name] - h * d})) / (2 * h)
    # (central differences: h^2 times a third derivative of order 10, and 1e-15 |loss| / h)
    assert abs(num - (b["d" + name] * d).sum()) < 1e-7 * max(1.0, abs(num))


def test_it_is_the_momentum_rule_without_momentum():
    x = inputs(3, H=3, Hk=3, dk=64, dv=64)
    f = gdr.forward(**x, scale=0.2)
    m = mdn_oracle.forward(x["q"], x["k"], x["v"], np.exp(x["g"]), x["beta"], np.zeros_like(x["beta"]), S0=x["S0"], scale=0.2)
    assert np.abs(f["o"] - m["o"]).max() < 1e-12 and np.abs(f["S"] - m["S"]).max() < 1e-12


def test_gates_at_their_limits():
    x = inputs(4)
    x["g"][:, 3] = -np.inf                       # forgets everything before
    x["beta"][:, 5] = 0.0                        # writes nothing
    f = gdr.forward(**x)
    tail = gdr.forward(**{n: (y[:, 3:] if n != "S0" else None) for n, y in x.items()})
    assert np.allclose(f["o"][:, 3:], tail["o"], atol=1e-14)
    dO = np.ones_like(x["v"])
    dO[:, :3] = 0.0
    b = gdr.backward(**x, dO=dO)
    assert (b["dg"][:, :4] == 0).all() and not b["dS0"].any() and np.isfinite(b["dbeta"]).all() and b["dbeta"][:, 5].any()
