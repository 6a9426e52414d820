"""CPU oracle for the feed-forward block around its FP8 linears.

TEST INFRASTRUCTURE ONLY: plain statements, in fp64 with numpy, of the layer
norm, the activations, the matmuls with a bias, an activation and a residual sum
after them, the gated pair of projections, and their gradients.  Operands are
values (already decoded); nothing here rounds, but for layernorm's h, which the
GPU path keeps in the tensor's type (the caller rounds it).
"""
from __future__ import annotations

import math

import numpy as np

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")   # FP8_ACT_* 0 .. 4
SLOPE_MAX = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "gelu_tanh": 1.13, "silu": 1.1}

_erfc = np.vectorize(math.erfc, otypes=[float])


def act(x, name):
    x = np.asarray(x, dtype=np.float64)
    if name == "relu":
        return np.where(x > 0, x, 0.0)
    if name == "gelu":
        return x * 0.5 * _erfc(-x / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + np.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    if name == "silu":
        return x / (1 + np.exp(-x))
    return x


def slope(x, name):
    x = np.asarray(x, dtype=np.float64)
    if name == "relu":
        return np.where(x > 0, 1.0, 0.0)
    if name == "gelu":
        return 0.5 * _erfc(-x / math.sqrt(2)) + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = np.tanh(k * (x + 0.044715 * x ** 3))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 3 * 0.044715 * x * x)
    if name == "silu":
        s = 1 / (1 + np.exp(-x))
        return s * (1 + x * (1 - s))
    return np.ones_like(x)


def linear_act(x, w, bias, name, res):
    """x [M, K], w [N, K]: (z, y)."""
    z = x @ w.T + (0 if bias is None else bias)
    return z, act(z, name) + (0 if res is None else res)


def linear_glu(x, w, bias, name):
    """w [2 N, K], gate rows first: (g | u) [M, 2 N] and a."""
    gu = x @ w.T + (0 if bias is None else bias)
    n = w.shape[0] // 2
    return gu, act(gu[:, :n], name) * gu[:, n:]


def linear_act_bwd(dy, w, z, name):
    """dy [M, N], w [K, N], z [M, K]: dz (its sum over rows is the bias gradient)."""
    return (dy @ w.T) * slope(z, name)


def linear_glu_bwd(dy, w, gu, name):
    """dy [M, N], w [K, N], gu [M, 2 K]: (dg | du)."""
    n = gu.shape[1] // 2
    t, g, u = dy @ w.T, gu[:, :n], gu[:, n:]
    return np.concatenate([t * u * slope(g, name), t * act(g, name)], axis=1)


def layernorm(h, g, b, eps):
    """(y, mean, rstd) of the rows of h."""
    mean = h.mean(axis=1)
    d = h - mean[:, None]
    rstd = 1 / np.sqrt((d * d).mean(axis=1) + eps)
    return d * rstd[:, None] * g + (0 if b is None else b), mean, rstd


def layernorm_bwd(dy, h, g, mean, rstd, dres=None):
    """(dx, dg, db)."""
    xh = (h - mean[:, None]) * rstd[:, None]
    w = dy * g
    dx = rstd[:, None] * (w - w.mean(axis=1, keepdims=True) - xh * (w * xh).mean(axis=1, keepdims=True))
    return dx + (0 if dres is None else dres), (dy * xh).sum(axis=0), dy.sum(axis=0)
