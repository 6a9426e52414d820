"""Pins of the feed-forward oracle against torch's autograd in fp64 (CPU), its limits, a row of equal
values, and which of the two projections is the gate.

fp64 on both sides: sums of at most 40 terms and a few functions, each within some ulps, so
1e-13 of the largest value is far above what rounding leaves (2^-53 * 40 * the terms' magnitudes
= 5e-15 of them) and far below any term's absence."""
import numpy as np
import pytest
import torch

from oracle import ffn as O

TORCH = {"none": lambda x: x, "relu": torch.relu, "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda x: torch.nn.functional.gelu(x, approximate="tanh"), "silu": torch.nn.functional.silu}


def leaf(r, *shape):
    return torch.from_numpy(r.normal(size=shape)).requires_grad_()


def same(got, want):
    want = want.detach().numpy() if isinstance(want, torch.Tensor) else want
    assert got.shape == want.shape
    assert np.max(np.abs(got - want)) <= 1e-13 * max(1.0, np.max(np.abs(want)))


@pytest.mark.parametrize("name", O.ACTS)
def test_activations(name):
    x = torch.linspace(-12, 12, 4801, dtype=torch.float64)
    x = x[x != 0].requires_grad_()  # torch's slope of ReLU at 0 is 0 too, but no derivative says so
    y = TORCH[name](x)
    y.sum().backward()
    same(O.act(x.detach().numpy(), name), y)
    same(O.slope(x.detach().numpy(), name), x.grad)


@pytest.mark.parametrize("name", [a for a in O.ACTS if a != "none"])
def test_limits(name):
    far = np.array([40.0, 300.0])
    assert np.allclose(O.act(far, name), far, rtol=1e-15) and np.allclose(O.slope(far, name), 1, rtol=1e-14)
    assert np.max(np.abs(O.act(-far, name))) < 2e-16 and np.max(np.abs(O.slope(-far, name))) < 2e-16


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("res", [False, True])
def test_layernorm(res, bias):
    r = np.random.default_rng(11)
    h, g, b, dy, dres = leaf(r, 5, 37), leaf(r, 37), leaf(r, 37), r.normal(size=(5, 37)), r.normal(size=(5, 37))
    y = torch.nn.functional.layer_norm(h, (37,), g, b if bias else None, 1e-3)
    ((y * torch.from_numpy(dy)).sum() + ((h * torch.from_numpy(dres)).sum() if res else 0)).backward()
    hv, gv, bv = (t.detach().numpy() for t in (h, g, b))
    got, mean, rstd = O.layernorm(hv, gv, bv if bias else None, 1e-3)
    same(got, y)
    same(mean, hv.mean(axis=1))
    same(rstd, 1 / np.sqrt(hv.var(axis=1) + 1e-3))
    dx, dg, db = O.layernorm_bwd(dy, hv, gv, mean, rstd, dres if res else None)
    same(dx, h.grad)
    same(dg, g.grad)
    if bias:
        same(db, b.grad)


def test_a_row_of_equal_values():
    y, mean, rstd = O.layernorm(np.full((2, 6), 3.0), np.full(6, 2.0), np.arange(6.0), 1e-4)
    assert np.array_equal(y, np.tile(np.arange(6.0), (2, 1))) and np.array_equal(mean, [3, 3]) and np.allclose(rstd, 100, rtol=1e-15)


@pytest.mark.parametrize("name", O.ACTS)
def test_linear(name):
    """Two linears with the activation between them: the second one's grad-input matmul, and the first one's bias gradient."""
    r = np.random.default_rng(12)
    x, w1, b1, w2, res, dy = leaf(r, 4, 3), leaf(r, 5, 3), leaf(r, 5), leaf(r, 6, 5), leaf(r, 4, 6), r.normal(size=(4, 6))
    z = x @ w1.t() + b1
    z.retain_grad()
    y = TORCH[name](z) @ w2.t() + res
    (y * torch.from_numpy(dy)).sum().backward()
    d = {k: v.detach().numpy() for k, v in dict(x=x, w1=w1, b1=b1, w2=w2, z=z, res=res).items()}
    zr, a = O.linear_act(d["x"], d["w1"], d["b1"], name, None)
    same(zr, z)
    same(a, TORCH[name](z))
    same(O.linear_act(a, d["w2"], None, "none", d["res"])[1], y)
    dz = O.linear_act_bwd(dy, d["w2"].T, zr, name)
    same(dz, z.grad)
    same(dz.sum(axis=0), b1.grad)


@pytest.mark.parametrize("name", O.ACTS)
def test_gated(name):
    """The gate's rows of w first: act of those, times the others."""
    r = np.random.default_rng(13)
    x, wg, wu, bias, wd, dy = leaf(r, 4, 3), leaf(r, 5, 3), leaf(r, 5, 3), leaf(r, 10), leaf(r, 6, 5), r.normal(size=(4, 6))
    g, u = x @ wg.t() + bias[:5], x @ wu.t() + bias[5:]
    g.retain_grad()
    u.retain_grad()
    a = TORCH[name](g) * u
    ((a @ wd.t()) * torch.from_numpy(dy)).sum().backward()
    d = {k: v.detach().numpy() for k, v in dict(x=x, wg=wg, wu=wu, bias=bias, wd=wd, a=a).items()}
    gu, got = O.linear_glu(d["x"], np.concatenate([d["wg"], d["wu"]]), d["bias"], name)
    same(gu, np.concatenate([g.detach().numpy(), u.detach().numpy()], axis=1))
    same(got, d["a"])
    dgu = O.linear_glu_bwd(dy, d["wd"].T, gu, name)
    same(dgu, np.concatenate([g.grad.numpy(), u.grad.numpy()], axis=1))
    same(dgu.sum(axis=0), bias.grad)
