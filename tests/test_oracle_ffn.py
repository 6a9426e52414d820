"""Pins of the feed-forward oracle (CPU): values by hand, and every gradient
against differences of the forward pass."""
import numpy as np
import pytest

from oracle import ffn as O

H = 1e-5
# A central difference is off by H^2/6 times the third derivative (below 20 for
# these functions and inputs: 3.4e-10) and by rounding, 2^-52 |f| / H (|f| < 100: 2.3e-9).
TOL = 4e-9


def test_activations_by_hand():
    assert O.act(0.0, "gelu") == 0 and O.act(0.0, "silu") == 0 and O.act(-1.0, "relu") == 0 and O.act(2.5, "relu") == 2.5
    assert np.isclose(O.act(1.0, "gelu"), 0.8413447460685429, rtol=1e-15)        # Phi(1)
    assert np.isclose(O.act(-3.0, "gelu"), -3 * 0.0013498980316300946, rtol=1e-14)
    assert np.isclose(O.act(1.0, "silu"), 0.7310585786300049, rtol=1e-15)        # 1 / (1 + 1/e)
    assert np.isclose(O.act(1.0, "gelu_tanh"), 0.841191990608276, rtol=1e-14)
    assert np.array_equal(O.slope(np.array([-1.0, 0.0, 1.0]), "relu"), [0, 0, 1])


@pytest.mark.parametrize("name", [a for a in O.ACTS if a != "relu"])
def test_slopes_are_the_differences(name):
    x = np.linspace(-8, 8, 401)
    assert np.max(np.abs((O.act(x + H, name) - O.act(x - H, name)) / (2 * H) - O.slope(x, name))) < TOL
    assert np.max(np.abs(O.slope(np.linspace(-30, 30, 10001), name))) <= O.SLOPE_MAX[name]


def differences(f, x):
    """Gradient of the scalar function f at x, by central differences."""
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = H
        out[i] = (f(x + e) - f(x - e)) / (2 * H)
    return out


@pytest.mark.parametrize("res", [False, True])
def test_layernorm_gradients_are_the_differences(res):
    r = np.random.default_rng(1)
    h, g, b, dy = r.normal(size=(3, 7)), 1 + 0.1 * r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    dres = r.normal(size=(3, 7)) if res else None
    y, mean, rstd = O.layernorm(h, g, b, 1e-5)
    assert np.allclose(((y - b) / g).mean(axis=1), 0, atol=1e-15) and np.allclose(((y - b) / g).var(axis=1), 1, atol=1e-4)
    dx, dg, db = O.layernorm_bwd(dy, h, g, mean, rstd, dres)
    extra = (lambda v: (v * dres).sum()) if res else (lambda v: 0.0)  # the stream that passes the norm by
    assert np.max(np.abs(differences(lambda v: (O.layernorm(v, g, b, 1e-5)[0] * dy).sum() + extra(v), h) - dx)) < TOL
    assert np.max(np.abs(differences(lambda v: (O.layernorm(h, v, b, 1e-5)[0] * dy).sum(), g) - dg)) < TOL
    assert np.max(np.abs(differences(lambda v: (O.layernorm(h, g, v, 1e-5)[0] * dy).sum(), b) - db)) < TOL


@pytest.mark.parametrize("name", [a for a in O.ACTS if a != "relu"])
def test_matmul_gradients_are_the_differences(name):
    r = np.random.default_rng(2)
    M, N, K = 3, 4, 5      # dy [M, N], w [K, N]: the linear after the activation
    dy, w = r.normal(size=(M, N)), r.normal(size=(K, N))
    z, gu = r.normal(size=(M, K)), r.normal(size=(M, 2 * K))
    loss = lambda v: ((O.act(v, name) @ w) * dy).sum()  # noqa: E731
    assert np.max(np.abs(differences(loss, z) - O.linear_act_bwd(dy, w, z, name))) < 4 * TOL
    loss = lambda v: (((O.act(v[:, :K], name) * v[:, K:]) @ w) * dy).sum()  # noqa: E731
    assert np.max(np.abs(differences(loss, gu) - O.linear_glu_bwd(dy, w, gu, name))) < 4 * TOL
    # the bias gradient: what a bias adds to every row
    bias = r.normal(size=K)
    loss = lambda v: ((O.act(z + v, name) @ w) * dy).sum()  # noqa: E731
    assert np.max(np.abs(differences(loss, bias) - O.linear_act_bwd(dy, w, z + bias, name).sum(axis=0))) < 8 * TOL


def test_forward_forms():
    r = np.random.default_rng(3)
    x, w, b, res = r.normal(size=(2, 3)), r.normal(size=(4, 3)), r.normal(size=4), r.normal(size=(2, 4))
    z, y = O.linear_act(x, w, b, "relu", res)
    assert np.allclose(z, x @ w.T + b) and np.allclose(y, np.maximum(z, 0) + res)
    gu, a = O.linear_glu(x, w, b, "none")
    assert np.allclose(a, gu[:, :2] * gu[:, 2:])
