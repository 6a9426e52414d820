"""The 256-row kernel of the feed-forward matmuls where it takes tiles 256 wide, alone and before a last round of tiles
64, 128 and 192 wide: what large outputs run.  On small whole numbers, where every sum
is exact, against torch in fp32 (exact there too): outputs, kept values, bias gradients,
codes and transposed codes, bit for bit."""
import ctypes

import pytest
import torch

import mm_routes as R
from paper_2309_17224_amd import fp8lin as F
from test_gpu_ffn import E4, E5, Strided, codes, ints, word

KINDS = ["act", "glu", "act_bwd", "glu_bwd"]
# rows, columns (of both projections, where the matmul is of both), contraction: (256-wide tiles there are, the others' width).
# Columns of a projection a multiple of eight (the codes are the epilogue's own), and odd ones.
SPLITS = {(2048, 8192, 384): (True, 0), (4090, 7696, 384): (True, 0), (4090, 4624, 384): (True, 64), (4090, 5392, 384): (True, 128),
          (4090, 6800, 384): (True, 192), (1030, 8208, 384): (False, 192)}
ODD = {(4090, 7698, 128): (True, 0), (4090, 4618, 128): (True, 64), (4090, 5398, 128): (True, 128), (4090, 6806, 128): (True, 192)}


def split(mode, M, N, K):
    """Tiles 256 wide, the width of the others and their number, of the output [M, N] (of one projection)."""
    f, v = R._lib().fp8lin_epi_split, [ctypes.c_int32() for _ in range(3)]
    f.argtypes = [ctypes.c_int32] + [ctypes.c_int64] * 3 + [ctypes.c_void_p] * 3
    return tuple(x.value for x in v) if f(mode, M, N, K, *map(ctypes.byref, v)) else None


def of(kind, shape):
    """Rows, columns (of one projection) and contraction; odd where half of the columns is."""
    M, cols, K = shape
    return M, cols // 2 if kind == "glu" else cols - (cols // 2) % 2, K


@pytest.mark.parametrize("kind", KINDS)
def test_shapes_take_every_split(kind):
    """No GPU needed."""
    seen = []
    for shape, want in {**SPLITS, **ODD}.items():
        M, N, K = of(kind, shape)
        got = split(KINDS.index(kind), M, N, K)
        assert got is not None and (got[0] > 0, got[1]) == want, (shape, got)
        assert (N % 8 == 0) == (shape in SPLITS) and (shape in SPLITS or N % 2 == 1)
        seen.append(want)
    assert {w for wide, w in seen if wide} == {0, 64, 128, 192}


def operands(kind, shape, gpu):
    M, N, K = of(kind, shape)
    gen = torch.Generator().manual_seed(M + 3 * N + len(kind))
    a8, a = codes(gen, M, K, E5 if "bwd" in kind else E4, gpu, True)
    b8, b = codes(gen, 2 * N if kind == "glu" else N, K, E4, gpu, True)
    t = torch.matmul(torch.from_numpy(a).float().to(gpu), torch.from_numpy(b).float().to(gpu).t().contiguous())
    assert float(t.abs().max()) < 2 ** 12
    side = ints(gen, M, 2 * N if kind == "glu_bwd" else N).to(gpu)
    return M, N, (a8, word(2, gpu), b8, word(-2, gpu)), t, side, ints(gen, 1, b8.shape[0])[0].to(gpu)


def run(kind, args, side, bias, M, N, gpu, fq=None):
    """The call with all that it writes in tensors between marks: outputs by name."""
    pad, off = (0, 0) if N % 8 == 0 else (3, 1)
    cols = 2 * N if kind == "glu_bwd" else N
    s = lambda c, v=None: Strided(M, c, torch.bfloat16, gpu, pad, off, v)  # noqa: E731
    out, db = s(cols), torch.empty(cols, device=gpu)
    if kind == "act":
        z = s(N)
        F.fp8_linear_fwd_act(*args, F.ACT_RELU, bias=bias, res=side, z=z.t, y=out.t, fq=fq)
        got = dict(out=out, z=z)
    elif kind == "glu":
        z = s(2 * N)
        F.fp8_linear_fwd_glu(*args, F.ACT_RELU, bias=bias, gu=z.t, a=out.t, fq=fq)
        got = dict(out=out, z=z)
    else:
        call = F.fp8_linear_bwd_dx_act if kind == "act_bwd" else F.fp8_linear_bwd_dx_glu
        call(*args, s(cols, side).t, F.ACT_RELU, out.t, db=db, fq=fq)
        got = dict(out=out, db=db)
    return got


def expected(kind, t, side, bias, N):
    """The same in fp32, unrounded."""
    if kind in ("act", "glu"):
        z = t + bias.float()
        y = z.clamp(min=0) + side.float() if kind == "act" else z[:, :N].clamp(min=0) * z[:, N:]
        return dict(out=y, z=z)
    v = side.float()
    if kind == "act_bwd":
        y = t * (v > 0)
    else:
        y = torch.cat([t * v[:, N:] * (v[:, :N] > 0), t * v[:, :N].clamp(min=0)], dim=1)
    assert float(y.abs().sum(dim=0).max()) < 2 ** 24     # every partial sum of a column is exact
    return dict(out=y, db=y.sum(dim=0, dtype=torch.float64).float())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", {**SPLITS, **ODD}, ids=str)
@pytest.mark.parametrize("kind", KINDS)
def test_outputs_exact(gpu, kind, shape):
    M, N, args, t, side, bias = operands(kind, shape, gpu)
    got, want = run(kind, args, side, bias, M, N, gpu), expected(kind, t, side, bias, N)
    for name, ref in want.items():
        if name == "db":
            assert torch.equal(got[name], ref), name
        else:
            assert torch.equal(got[name].t, ref.to(torch.bfloat16)) and got[name].untouched(), name


@pytest.mark.gpu
@pytest.mark.parametrize("shape", {**SPLITS, **ODD}, ids=str)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("off", [0, 1])
def test_codes(gpu, kind, shape, off):
    """Of a prediction that holds, and of one that is off by one."""
    M, N, args, t, side, bias = operands(kind, shape, gpu)
    want = expected(kind, t, side, bias, N)
    y = want["out"].to(torch.bfloat16)
    fmt, cols = F.E5M2 if "bwd" in kind else F.E4M3, y.shape[1]
    q, qT, b, amax, flags = F.fp8_quantise(y, fmt, 0, want_qT=True)
    qs, qTs = Strided(M, cols, torch.uint8, gpu, 3, 1), Strided(cols, M, torch.uint8, gpu, 5, 2)
    ws = torch.empty(F.fp8_linear_quantise_ws_bytes(M, cols), dtype=torch.uint8, device=gpu)
    fq = F.FusedQuant(qs.t, word(-99, gpu), ws, fmt, bias_pred=word(int(b) + off, gpu), amax_bits=word(-99, gpu),
                      flags=word(-99, gpu), qT=qTs.t)
    got = run(kind, args, side, bias, M, N, gpu, fq)
    assert torch.equal(got["out"].t, y)
    assert (int(fq.bias), int(fq.amax_bits), int(fq.flags)) == (int(b), int(amax), int(flags))
    assert torch.equal(qs.t, q) and qs.untouched()
    assert torch.equal(qTs.t, qT) and qTs.untouched()
    if "db" in want:
        assert torch.equal(got["db"], want["db"])
