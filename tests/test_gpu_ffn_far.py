"""The feed-forward calls where offsets pass 32 bits: rows of 2^22 elements and more
apart (up to 2^22 the 256-row kernel's lanes hold their offsets in 32 bits), a few
rows of 2^30, more rows or columns than a launch has workgroups.  On whole numbers
every output equals that of the same call on dense tensors, bit for bit."""
import pytest
import torch

import mm_routes as R
from paper_2309_17224_amd import fp8lin as F
from test_gpu_ffn import E4, E5, codes, ints, word

pytestmark = pytest.mark.gpu

LD = [1 << 22, (1 << 22) + 8]
FAR = {"small": ((5, 40, 128), [1 << 30]), "any k": ((5, 40, 130), [1 << 30]), "256": ((1030, 8200, 256), LD)}
KINDS = {"act": 0, "glu": 1, "act_bwd": 2, "glu_bwd": 3}


def far(rows, cols, ld, dtype, gpu, value=None):
    t = torch.empty(rows * ld, dtype=dtype, device=gpu).view(rows, ld)[:, :cols]
    if value is not None:
        t.copy_(value)
    return t


def quant(rows, cols, fmt, gpu, ld=None, ldT=None):
    return F.FusedQuant(far(rows, cols, ld or cols, torch.uint8, gpu), word(0, gpu),
                        torch.empty(F.fp8_linear_quantise_ws_bytes(rows, cols), dtype=torch.uint8, device=gpu), fmt,
                        bias_pred=word(1, gpu), amax_bits=word(0, gpu), qT=far(cols, rows, ldT or rows, torch.uint8, gpu))


def same_codes(a, b):
    assert int(a.bias) == int(b.bias) and int(a.amax_bits) == int(b.amax_bits)
    assert torch.equal(a.q, b.q) and torch.equal(a.qT, b.qT)


def test_shapes_take_the_kernels_named():
    for mode in range(4):
        assert R.epilogue(mode, *FAR["small"][0])[0] == R.STREAM
        assert R.epilogue(mode, *FAR["any k"][0])[0] == R.RAGGED
        assert R.epilogue(mode, *FAR["256"][0])[0] == R.MAIN
        assert R.epilogue(mode, 16400, 520, 128)[0] == R.MAIN


@pytest.mark.parametrize("route,ld", [(r, ld) for r, (_, lds) in FAR.items() for ld in lds])
@pytest.mark.parametrize("kind", KINDS)
def test_rows_far_apart(gpu, route, ld, kind):
    M, N, K = FAR[route][0]
    gen = torch.Generator().manual_seed(N + len(kind))
    a8, _ = codes(gen, M, K, E5 if "bwd" in kind else E4, gpu, True)
    b8, _ = codes(gen, 2 * N if kind == "glu" else N, K, E4, gpu, True)
    one, fmt, wide = word(0, gpu), F.E5M2 if "bwd" in kind else F.E4M3, 2 * N if "glu" in kind else N
    side = ints(gen, M, wide if "bwd" in kind else N).to(gpu)
    cols = wide if kind == "glu_bwd" else N
    dense, apart = quant(M, cols, fmt, gpu), quant(M, cols, fmt, gpu, ld=ld)
    bf, out = torch.bfloat16, far(M, cols, ld, torch.bfloat16, gpu)
    if "bwd" in kind:
        call = F.fp8_linear_bwd_dx_act if kind == "act_bwd" else F.fp8_linear_bwd_dx_glu
        db, db2 = torch.empty(cols, device=gpu), torch.empty(cols, device=gpu)
        want = call(a8, one, b8, one, side, F.ACT_RELU, db=db, fq=dense)
        call(a8, one, b8, one, far(M, wide, ld, bf, gpu, side), F.ACT_RELU, out, db=db2, fq=apart)
        assert torch.equal(db, db2)
    else:
        keep, keep2 = torch.empty(M, wide, dtype=bf, device=gpu), far(M, wide, ld, bf, gpu)
        if kind == "act":
            want = F.fp8_linear_fwd_act(a8, one, b8, one, F.ACT_RELU, res=side, z=keep, fq=dense)
            F.fp8_linear_fwd_act(a8, one, b8, one, F.ACT_RELU, res=far(M, N, ld, bf, gpu, side), z=keep2, y=out, fq=apart)
        else:
            want = F.fp8_linear_fwd_glu(a8, one, b8, one, F.ACT_RELU, gu=keep, fq=dense)
            F.fp8_linear_fwd_glu(a8, one, b8, one, F.ACT_RELU, gu=keep2, a=out, fq=apart)
        assert torch.equal(keep, keep2)
    assert torch.equal(out, want) and torch.count_nonzero(want) > 0
    same_codes(apart, dense)


@pytest.mark.parametrize("ld", LD)
@pytest.mark.parametrize("kind", KINDS)
def test_transposed_codes_far_apart(gpu, ld, kind):
    M, N, K = 16400, 520, 128
    gen = torch.Generator().manual_seed(len(kind))
    a8, _ = codes(gen, M, K, E5 if "bwd" in kind else E4, gpu, True)
    b8, _ = codes(gen, 2 * N if kind == "glu" else N, K, E4, gpu, True)
    one, fmt = word(0, gpu), F.E5M2 if "bwd" in kind else F.E4M3
    cols = 2 * N if kind == "glu_bwd" else N
    side = ints(gen, M, cols).to(gpu)
    dense, apart = quant(M, cols, fmt, gpu), quant(M, cols, fmt, gpu, ldT=ld)
    for fq in (dense, apart):
        if kind == "act":
            F.fp8_linear_fwd_act(a8, one, b8, one, F.ACT_RELU, fq=fq)
        elif kind == "glu":
            F.fp8_linear_fwd_glu(a8, one, b8, one, F.ACT_RELU, fq=fq)
        elif kind == "act_bwd":
            F.fp8_linear_bwd_dx_act(a8, one, b8, one, side, F.ACT_RELU, fq=fq)
        else:
            F.fp8_linear_bwd_dx_glu(a8, one, b8, one, side, F.ACT_RELU, fq=fq)
    same_codes(apart, dense)


@pytest.mark.parametrize("rows,cols,ld", [(5, 40, 1 << 30), (1100, 1032, 1 << 22)])
def test_norm_and_bias_grad_of_rows_far_apart(gpu, rows, cols, ld):
    bf = torch.bfloat16
    gen = torch.Generator().manual_seed(rows)
    x, res, dy = (torch.randn(rows, cols, generator=gen).to(bf).to(gpu) for _ in range(3))
    g = torch.randn(cols, generator=gen).to(gpu)
    f32 = lambda: torch.empty(rows, device=gpu)  # noqa: E731
    h, mean, rstd, h2, mean2, rstd2 = torch.empty_like(x), f32(), f32(), far(rows, cols, ld, bf, gpu), f32(), f32()
    y = F.gpt_layernorm_quantise(x, g, res=res, h=h, mean=mean, rstd=rstd)
    y2 = far(rows, cols, ld, bf, gpu)
    F.gpt_layernorm_quantise(far(rows, cols, ld, bf, gpu, x), g, res=far(rows, cols, ld, bf, gpu, res), h=h2, y=y2, mean=mean2,
                             rstd=rstd2)
    for a, b in ((y, y2), (h, h2), (mean, mean2), (rstd, rstd2)):
        assert torch.equal(a, b)
    want = F.gpt_layernorm_bwd(dy, h, g, mean, rstd, dres=res)
    dyf = far(rows, cols, ld, bf, gpu, dy)
    got = F.gpt_layernorm_bwd(dyf, h2, g, mean, rstd, dres=far(rows, cols, ld, bf, gpu, res), dx=y2)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    assert torch.equal(F.gpt_bias_grad(dyf), F.gpt_bias_grad(dy))


def test_norm_of_more_rows_than_a_launch_has(gpu):
    rows, cols, k = (1 << 23) + 5, 1032, 64
    gen = torch.Generator().manual_seed(1)
    some = torch.randn(k, cols, generator=gen).to(torch.bfloat16).to(gpu)
    g = torch.randn(cols, generator=gen).to(gpu)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=gpu)
    x[:rows // k * k].view(-1, k, cols).copy_(some)
    x[rows // k * k:] = some[:rows % k]
    last = some[:1] * 0
    last[0, 5] = 1                    # a row of its own, with the largest output: (cols - 1) / sqrt(cols)
    g[5] = 4.0
    x[-1:] = last
    mean, rstd = torch.empty(rows, device=gpu), torch.empty(rows, device=gpu)
    fq = F.FusedQuant(torch.empty((rows, cols), dtype=torch.uint8, device=gpu), word(0, gpu),
                      torch.empty(F.gpt_layernorm_ws_bytes(rows), dtype=torch.uint8, device=gpu), F.E4M3, bias_pred=word(1, gpu),
                      amax_bits=word(0, gpu))
    y = F.gpt_layernorm_quantise(x, g, mean=mean, rstd=rstd, fq=fq)
    few = torch.cat([some, last])
    m2, r2 = torch.empty(k + 1, device=gpu), torch.empty(k + 1, device=gpu)
    want = F.gpt_layernorm_quantise(few, g, mean=m2, rstd=r2)
    q, _, bias, amax, _ = F.fp8_quantise(want, F.E4M3, 0)
    assert int(fq.bias) == int(bias) and int(fq.amax_bits) == int(amax)
    for got, of in ((y, want), (mean, m2), (rstd, r2), (fq.q, q)):
        n = rows // k
        assert bool((got[:n * k].view(n, k, -1) == of[:k].view(1, k, -1)).all())
        assert torch.equal(got[n * k:-1], of[:rows - 1 - n * k]) and torch.equal(got[-1:], of[k:])


def test_sums_of_more_columns_than_a_launch_has(gpu):
    cols = (1 << 22) + 70
    gen = torch.Generator().manual_seed(2)
    dy = ints(gen, 3, cols).to(gpu)
    assert torch.equal(F.gpt_bias_grad(dy), dy.float().sum(dim=0))
    w8, w = codes(gen, cols, 1, E4, gpu, True)
    dy8, d = codes(gen, 2, 1, E5, gpu, True)
    db = torch.empty(cols, device=gpu)
    z = ints(gen, 2, cols).to(gpu)
    dz = F.fp8_linear_bwd_dx_act(dy8, word(0, gpu), w8, word(0, gpu), z, F.ACT_RELU, db=db)
    want = torch.from_numpy(d @ w.T).to(gpu) * (z > 0)
    assert torch.equal(dz.double(), want) and torch.equal(db.double(), want.sum(dim=0))
