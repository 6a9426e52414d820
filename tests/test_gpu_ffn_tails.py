"""The activations and their slopes far out, relative to their own size: all four
matmuls, in small tiles and in 256-row tiles, of zero operands (the bias is then the
value before the activation) or of operands whose product is 1.

Bars, from the arithmetic.  Each form is one exponential 2^-p: p is off by at most 3.5
roundings, 3.5 |p| 2^-24, which its exponential passes on times ln 2; with the fit of the
Gauss tail (6e-7), the exponential's and the reciprocal's last bit and four products that
is below (1 + |p| / 4) 2^-20 of the value.  A slope is a sum of two terms, each of which
is off by that.  Below 2^-126 an exponential or a reciprocal may be 0: then |x| 2^-125
(a slope's second term, x p' times that) is lost.  Then half a step of the output's type.
"""
import math

import numpy as np
import pytest
import torch

import mm_routes as R
from paper_2309_17224_amd import fp8lin as F
from test_gpu_ffn import ACT, E4, E5, HALF, word

pytestmark = pytest.mark.gpu

ACTS = ["gelu", "gelu_tanh", "silu"]
N, K = 4104, 128
ROWS = {"small tiles": (5, R.STREAM), "256-row tiles": (700, R.MAIN)}
INF = float("inf")
FAR = [-INF, -3e38, -1e4, -200.0]           # 0, and no slope
LIMIT = [200.0, 1e4, 3e38, INF]             # x, and slope 1


def forms(x, name):
    """act, slope, the magnitude of the slope's two terms, |p| of the exponential 2^-p, |x p'| ln 2; in fp64."""
    if name == "gelu":
        phi = np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        cdf = 0.5 * np.vectorize(math.erfc)(-x / math.sqrt(2))
        return x * cdf, cdf + x * phi, cdf + np.abs(x) * phi, x * x / 2 / math.log(2), np.abs(x)
    c = 2 * math.sqrt(2 / math.pi)
    u = x if name == "silu" else c * (x + 0.044715 * x ** 3)
    d = 1.0 if name == "silu" else c * (1 + 3 * 0.044715 * x * x)
    s, r = 1 / (1 + np.exp(-u)), 1 / (1 + np.exp(u))
    return x * s, s * (1 + x * d * r), s * (1 + np.abs(x * d) * r), np.abs(u) / math.log(2), np.abs(x * d)


def points():
    """Values of bf16: both signs, close together where a tail has its last normal values."""
    g = np.random.default_rng(5)
    x = np.concatenate([-np.exp(g.uniform(np.log(1e-3), np.log(95), 2600)), -g.uniform(5, 14, 900), g.uniform(0, 95, 500)])
    x = torch.from_numpy(np.concatenate([FAR, LIMIT, [float("nan")], x, np.zeros(N - 9 - len(x))])).to(torch.bfloat16)
    x[0:8] = torch.tensor(FAR + LIMIT).to(torch.bfloat16)
    return x


def held(got, ref, err, dt, name):
    """All rows alike, the first one's finite points within err and half a step, the others their limits."""
    got = got.cpu()
    assert torch.equal(got[1:].nan_to_num(1.5, 2.5, 3.5), got[:1].expand_as(got[1:]).nan_to_num(1.5, 2.5, 3.5))
    g = got[0].double().numpy()
    assert np.array_equal(g[:4], np.zeros(4)), g[:4]
    assert math.isnan(g[8])
    g, ref, err = g[9:], ref[9:], err[9:]
    off = np.abs(g - ref) - (err + HALF[dt] * (np.abs(ref) + err) + 2.0 ** -149)
    worst = int(np.argmax(off))
    assert off[worst] <= 0, (name, worst, g[worst], ref[worst], err[worst])
    return got[0, 4:8]


def reference(act):
    x = points()
    with np.errstate(all="ignore"):
        f, d, terms, p, xp = forms(x.double().numpy(), act)
        rel = (1 + p / 4) * 2.0 ** -20
        xs = np.abs(x.double().numpy())
        return x, f, rel * np.abs(f) + xs * 2.0 ** -125, d, rel * terms + (1 + xp) * 2.0 ** -125


def ones(rows, cols, kind, gpu):
    return torch.ones((rows, cols), device=gpu).to(kind).view(torch.uint8)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("act", ACTS)
def test_values(gpu, rows, act):
    M, kernel = ROWS[rows]
    assert R.epilogue(0, M, N, K)[0] == R.epilogue(1, M, N, K)[0] == kernel
    x, f, ef, _, _ = reference(act)
    limit = torch.tensor(LIMIT).to(torch.bfloat16)
    zero = lambda r: torch.zeros((r, K), dtype=torch.uint8, device=gpu)  # noqa: E731
    for dt in (torch.float32, torch.bfloat16):
        y = F.fp8_linear_fwd_act(zero(M), word(0, gpu), zero(N), word(0, gpu), ACT[act], bias=x.to(gpu),
                                 out_dt=F.DT_F32 if dt is torch.float32 else F.DT_BF16)
        assert torch.equal(held(y, f, ef, dt, act).to(torch.bfloat16), limit)
    both = torch.cat([x, torch.ones(N, dtype=torch.bfloat16)]).to(gpu)
    a = F.fp8_linear_fwd_glu(zero(M), word(0, gpu), zero(2 * N), word(0, gpu), ACT[act], bias=both)
    assert torch.equal(held(a, f, ef, torch.bfloat16, act), limit)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("act", ACTS)
def test_slopes(gpu, rows, act):
    M, kernel = ROWS[rows]
    assert R.epilogue(2, M, N, K)[0] == R.epilogue(3, M, N, K)[0] == kernel
    x, f, ef, d, ed = reference(act)
    dy, w = ones(M, K, E5, gpu), ones(N, K, E4, gpu)
    z = x.expand(M, N).contiguous().to(gpu)
    dz = F.fp8_linear_bwd_dx_act(dy, word(3, gpu), w, word(4, gpu), z, ACT[act])   # t = 1
    assert torch.equal(held(dz, d, ed, torch.bfloat16, act), torch.ones(4, dtype=torch.bfloat16))
    gu = torch.cat([z, torch.ones_like(z)], dim=1)
    dgu = F.fp8_linear_bwd_dx_glu(dy, word(3, gpu), w, word(4, gpu), gu, ACT[act])
    assert torch.equal(held(dgu[:, :N], d, ed, torch.bfloat16, act), torch.ones(4, dtype=torch.bfloat16))
    assert torch.equal(held(dgu[:, N:], f, ef, torch.bfloat16, act), torch.tensor(LIMIT).to(torch.bfloat16))
