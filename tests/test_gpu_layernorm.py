"""Layer norm forward and backward and the bias gradient against the oracle in fp64.

Bars, from the arithmetic.  A sum of n fp32 terms taken by up to 2048 threads,
each at most 8 of them in a row (more for rows beyond 16384 columns: n / 2048), then
through a tree of at most 16 levels, is off by at most S(n) = (n / 2048 + 24) 2^-24
of the sum of magnitudes.  The mean is thus off by S mean|h|, and so is every
centred value, plus its own rounding; the variance by 2 S of itself and the square
of the mean's error; rstd by half of that and two roundings; the products of the
output round four more times.  Then half a step of the output's type.  The column sums
add at most R = rows / slots values in a row and then the slots' sums."""
import numpy as np
import pytest
import torch

from oracle import ffn as O
from paper_2309_17224_amd import fp8lin as F
from test_gpu_ffn import Strided, close, word

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5
# rows x columns: one element, single rows, odd widths, each width class of the kernels and its borders, wider than registers
SIZES = [(1, 1), (1, 768), (7, 3), (3, 512), (5, 513), (70, 1023), (9, 1032), (6, 2049), (13, 4096), (4, 4104), (5, 8192),
         (3, 8200), (3, 16384), (3, 16392), (2, 20011)]


def S(n):
    return (n / 2048 + 24) * U


def data(rows, cols, dt, seed, mean=0.3):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, cols, generator=gen) + mean).to(dt)
    g, b = (1 + 0.1 * torch.randn(cols, generator=gen)), 0.1 * torch.randn(cols, generator=gen)
    return gen, x, g, b


def stat_errors(h, mean, rstd):
    """Bounds of the errors of the mean and (relative) of rstd."""
    n = h.shape[1]
    dm = S(n) * np.abs(h).mean(axis=1) + U * np.abs(mean)
    var = ((h - mean[:, None]) ** 2).mean(axis=1)
    # centred values: the mean's error and their rounding; their squares' mean
    d = dm + U * np.abs(h - mean[:, None]).max(axis=1)
    dv = (2 * S(n) + 4 * U) * var + 2 * d * np.sqrt(var) + d * d
    return dm, 0.5 * dv * rstd ** 2 / np.maximum(1e-30, 1 - dv * rstd ** 2) + 4 * U


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("res,gdt,pad,off", [(False, torch.bfloat16, 0, 0), (True, torch.float32, 5, 1)])
def test_forward(gpu, size, dt, res, gdt, pad, off):
    rows, cols = size
    gen, x, g, b = data(rows, cols, dt, 31 * rows + cols)
    g, b = g.to(gdt), b.to(gdt)
    r = torch.randn(rows, cols, generator=gen).to(dt) if res else None
    h = (x.float() + r.float()).to(dt) if res else x      # the fp32 sum of two bf16 or fp32 values, rounded once
    bb = b if res or cols % 2 else None
    xs, ys, hs = (Strided(rows, cols, dt, gpu, pad, off, v) for v in (x.to(gpu), None, None))
    rs = Strided(rows, cols, dt, gpu, pad + 2, off, r.to(gpu)) if res else None
    mean, rstd = torch.empty(rows, device=gpu), torch.empty(rows, device=gpu)
    F.gpt_layernorm_quantise(xs.t, g.to(gpu), None if bb is None else bb.to(gpu), EPS, res=rs.t if res else None, h=hs.t,
                             y=ys.t, mean=mean, rstd=rstd)
    assert torch.equal(hs.t.cpu(), h) and hs.untouched() and ys.untouched()
    hv, gv = h.double().numpy(), g.double().numpy()
    y, m, s = O.layernorm(hv, gv, 0 if bb is None else bb.double().numpy(), EPS)
    dm, ds = stat_errors(hv, m, s)
    close(mean, m, dm, torch.float32)
    close(rstd, s, ds * s, torch.float32)
    xh = np.abs(hv - m[:, None]) * s[:, None]
    err = np.abs(gv) * (xh * (ds[:, None] + 4 * U) + dm[:, None] * s[:, None]) + 2 * U * (np.abs(y) + np.abs(gv) * xh)
    close(ys.t, y, err, dt)
    # the same without the optional outputs
    y2 = F.gpt_layernorm_quantise(xs.t, g.to(gpu), None if bb is None else bb.to(gpu), EPS, res=rs.t if res else None)
    assert torch.equal(y2, ys.t)


# rows by waves and by blocks, on both sides of each border
@pytest.mark.parametrize("size", [(768, 1000), (769, 521), (1999, 1031), (2000, 1283), (2003, 2048), (2999, 2056), (3000, 2560),
                                  (3001, 2051), (3000, 2561)], ids=str)
@pytest.mark.parametrize("dt,res,gdt,pad,off", [(torch.bfloat16, True, torch.bfloat16, 3, 1), (torch.float32, False, torch.float32, 0, 0)])
def test_forward_of_many_rows(gpu, size, dt, res, gdt, pad, off):
    test_forward(gpu, size, dt, res, gdt, pad, off)


@pytest.mark.parametrize("size", [(770, 1000), (2001, 1290), (3001, 2104)], ids=str)
def test_codes_of_many_rows(gpu, size):
    for pred in (None, 0, 1):
        test_codes_are_those_of_the_output(gpu, size, pred, F.E4M3)


@pytest.mark.parametrize("cols", [500, 768, 1001, 1283, 2048, 2560, 5000])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_a_row_is_the_same_in_any_batch(gpu, cols, dt):
    _, x, g, b = data(3001, cols, dt, cols)
    x, g, b = x.to(gpu), g.to(gpu), b.to(gpu)
    seen = []
    for n in (3, 768, 769, 1999, 2000, 3001):
        mean, rstd = torch.empty(n, device=gpu), torch.empty(n, device=gpu)
        seen.append((F.gpt_layernorm_quantise(x[:n], g, b, mean=mean, rstd=rstd)[:3], mean[:3], rstd[:3]))
    for other in seen[1:]:
        assert all(torch.equal(p, q) for p, q in zip(seen[0], other))


@pytest.mark.parametrize("size", SIZES + [(300, 96), (1111, 1024), (600, 640)], ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("res,gdt,pad,off", [(False, torch.float32, 0, 0), (True, torch.bfloat16, 3, 1)])
def test_backward(gpu, size, dt, res, gdt, pad, off):
    rows, cols = size
    gen, h, g, _ = data(rows, cols, dt, 17 * rows + cols)
    g = g.to(gdt)
    dy = torch.randn(rows, cols, generator=gen).to(dt)
    dres = torch.randn(rows, cols, generator=gen).to(dt) if res else None
    hv, gv, dyv = h.double().numpy(), g.double().numpy(), dy.double().numpy()
    _, m, s = O.layernorm(hv, gv, None, EPS)
    mean, rstd = torch.from_numpy(m).float(), torch.from_numpy(s).float()
    m, s = mean.double().numpy(), rstd.double().numpy()  # the call's inputs
    dx, dg, db = O.layernorm_bwd(dyv, hv, gv, m, s, dres.double().numpy() if res else None)
    hs, dys, dxs = (Strided(rows, cols, dt, gpu, pad, off, v) for v in (h.to(gpu), dy.to(gpu), None))
    rs = Strided(rows, cols, dt, gpu, pad + 1, off, dres.to(gpu)) if res else None
    sums = torch.full((2 * cols + 4,), 7.0, device=gpu)
    args = (dys.t, hs.t, g.to(gpu), mean.to(gpu), rstd.to(gpu))
    F.gpt_layernorm_bwd(*args, dres=rs.t if res else None, dx=dxs.t, dg=sums[1:1 + cols], db=sums[2 + cols:2 + 2 * cols])
    # xh: a rounded difference times rstd; w: a product; the two means: S of the magnitudes
    xh, w = (hv - m[:, None]) * s[:, None], dyv * gv
    c1, c2 = np.abs(w).mean(axis=1)[:, None], np.abs(w * xh).mean(axis=1)[:, None]
    n = S(cols) + 6 * U
    err = s[:, None] * (n * (c1 + np.abs(xh) * c2) + 6 * U * (np.abs(w) + c1 + np.abs(xh) * c2))
    close(dxs.t, dx, err + U * (np.abs(dx) + (np.abs(dres.double().numpy()) if res else 0)), dt)
    assert dxs.untouched()
    add = (rows + 24) * U                                # any order of the rows' sums
    close(sums[1:1 + cols], dg, (add + 3 * U) * (np.abs(dyv * xh)).sum(axis=0), torch.float32)
    close(sums[2 + cols:2 + 2 * cols], db, add * np.abs(dyv).sum(axis=0), torch.float32)
    assert float(sums[0]) == float(sums[1 + cols]) == float(sums[2 + 2 * cols]) == 7.0
    # only one of the two, or neither; the same bits every time
    dx2, dg2, db2 = F.gpt_layernorm_bwd(*args, dres=rs.t if res else None)
    assert torch.equal(dx2, dxs.t) and torch.equal(dg2, sums[1:1 + cols]) and torch.equal(db2, sums[2 + cols:2 + 2 * cols])
    dx3, dg3, none = F.gpt_layernorm_bwd(*args, dres=rs.t if res else None, dg=torch.empty(cols, device=gpu), want_params=False)
    assert none is None and torch.equal(dg3, dg2) and torch.equal(dx3, dx2)
    assert F.gpt_layernorm_bwd(*args, want_params=False)[1:] == (None, None)


def test_a_large_mean(gpu):
    """A mean of 1000 times the spread: the variance is of the centred values."""
    rows, cols = 4, 5120
    gen = torch.Generator().manual_seed(3)
    x = (torch.randn(rows, cols, generator=gen) + 1000).float()
    mean, rstd = torch.empty(rows, device=gpu), torch.empty(rows, device=gpu)
    y = F.gpt_layernorm_quantise(x.to(gpu), torch.ones(cols, device=gpu), eps=0.0, mean=mean, rstd=rstd)
    ref, m, s = O.layernorm(x.double().numpy(), 1.0, 0.0, 0.0)
    dm, ds = stat_errors(x.double().numpy(), m, s)
    close(mean, m, dm, torch.float32)
    close(rstd, s, ds * s, torch.float32)
    close(y, ref, np.abs(ref) * (ds[:, None] + 4 * U) + dm[:, None] * s[:, None], torch.float32)


def test_constant_and_nonfinite_rows(gpu):
    """A constant row has variance 0: y = b.  NaN and infinity stay in their rows."""
    x = torch.full((4, 300), 3.0)
    x[1, 5], x[2, 7] = float("nan"), float("inf")
    g, b = torch.full((300,), 2.0), torch.arange(300.0)
    y = F.gpt_layernorm_quantise(x.to(gpu), g.to(gpu), b.to(gpu), EPS).cpu()
    assert torch.equal(y[0], b) and torch.equal(y[3], b)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()


@pytest.mark.parametrize("size", [(1, 8), (33, 768), (300, 520), (5, 5120), (3, 16400), (9, 37)], ids=str)
@pytest.mark.parametrize("pred", [None, 0, 1, -2, "alias"])
@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2, F.E4_A])
def test_codes_are_those_of_the_output(gpu, size, pred, fmt):
    rows, cols = size
    gen, x, g, b = data(rows, cols, torch.bfloat16, cols)
    x, g, b = x.to(gpu), g.to(gpu), b.to(gpu)
    alone = F.gpt_layernorm_quantise(x, g, b)
    q, _, bias, amax, flags = F.fp8_quantise(alone, fmt, 1)
    bs = word(int(bias) - 3, gpu)
    p = None if pred is None else bs if pred == "alias" else word(int(bias) + pred, gpu)
    qs = Strided(rows, cols, torch.uint8, gpu, 3, 1)
    fq = F.FusedQuant(qs.t, bs, torch.empty(F.gpt_layernorm_ws_bytes(rows), dtype=torch.uint8, device=gpu), fmt, 1, bias_pred=p,
                      amax_bits=word(0, gpu), flags=word(9, gpu))
    assert torch.equal(F.gpt_layernorm_quantise(x, g, b, fq=fq), alone)
    assert torch.equal(qs.t, q) and qs.untouched()
    assert (int(bs), int(fq.amax_bits), int(fq.flags)) == (int(bias), int(amax), int(flags))


@pytest.mark.parametrize("size", [(1, 1), (3, 8), (64, 512), (65, 513), (1000, 37), (4097, 768), (20000, 24)], ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_bias_grad(gpu, size, dt):
    rows, cols = size
    gen = torch.Generator().manual_seed(rows)
    dy = torch.randn(rows, cols, generator=gen).to(dt)
    d = Strided(rows, cols, dt, gpu, 3, 1, dy.to(gpu))
    ref, mags = dy.double().numpy().sum(axis=0), np.abs(dy.double().numpy()).sum(axis=0)
    db = F.gpt_bias_grad(d.t)
    close(db, ref, (rows + 24) * U * mags, torch.float32)
    half = F.gpt_bias_grad(d.t, db=torch.empty(cols, dtype=torch.bfloat16, device=gpu))
    assert torch.equal(half, db.to(torch.bfloat16))
    whole = torch.randint(-4, 5, (rows, cols), generator=gen).to(dt)   # sums below 2^24: exact
    assert torch.equal(F.gpt_bias_grad(whole.to(gpu)).cpu(), whole.double().sum(dim=0).float())


def test_empty(gpu):
    e = lambda *s: torch.empty(s, device=gpu)  # noqa: E731
    dx, dg, db = F.gpt_layernorm_bwd(e(0, 9), e(0, 9), torch.ones(9, device=gpu), e(0), e(0))
    assert dx.shape == (0, 9) and torch.equal(dg, torch.zeros(9, device=gpu)) and torch.equal(db, torch.zeros(9, device=gpu))
    assert torch.equal(F.gpt_bias_grad(e(0, 5)), torch.zeros(5, device=gpu))
    assert F.gpt_layernorm_quantise(e(0, 9), torch.ones(9, device=gpu)).shape == (0, 9)
    b, fl = word(5, gpu), word(5, gpu)
    fq = F.FusedQuant(torch.empty((0, 8), dtype=torch.uint8, device=gpu), b, torch.empty(4, dtype=torch.uint8, device=gpu), flags=fl)
    F.gpt_layernorm_quantise(torch.empty((0, 8), dtype=torch.bfloat16, device=gpu), torch.ones(8, device=gpu), fq=fq)
    assert int(b) == 0 and int(fl) == F.FLAG_ZERO


def test_binding_refuses(gpu):
    x = torch.zeros((4, 8), dtype=torch.bfloat16, device=gpu)
    v, s = torch.zeros(8, device=gpu), torch.zeros(4, device=gpu)
    fq = F.FusedQuant(torch.zeros((4, 8), dtype=torch.uint8, device=gpu), word(0, gpu),
                      torch.zeros(64, dtype=torch.uint8, device=gpu), qT=torch.zeros((8, 4), dtype=torch.uint8, device=gpu))
    bad = [(TypeError, lambda: F.gpt_layernorm_quantise(x.half(), v)), (ValueError, lambda: F.gpt_layernorm_quantise(x, v[:7])),
           (TypeError, lambda: F.gpt_layernorm_quantise(x, v, v.to(torch.bfloat16))),
           (TypeError, lambda: F.gpt_layernorm_quantise(x, v, res=x.float())),
           (ValueError, lambda: F.gpt_layernorm_quantise(x, v, mean=v)), (ValueError, lambda: F.gpt_layernorm_quantise(x.t(), v)),
           (F.Fp8Error, lambda: F.gpt_layernorm_quantise(x, v, fq=fq)), (F.Fp8Error, lambda: F.gpt_layernorm_quantise(x, v, eps=-1.0)),
           (TypeError, lambda: F.gpt_layernorm_bwd(x, x.float(), v, s, s)), (ValueError, lambda: F.gpt_layernorm_bwd(x, x, v, v, s)),
           (F.Fp8Error, lambda: F.gpt_layernorm_bwd(x, x, v, s, s, ws=torch.zeros(4, dtype=torch.uint8, device=gpu)))]
    for error, fn in bad:
        with pytest.raises(error):
            fn()
