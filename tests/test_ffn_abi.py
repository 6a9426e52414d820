"""The feed-forward calls on the host (no GPU needed): every refusal comes before
anything would be launched."""
import ctypes
import os

import pytest
import torch

from paper_2309_17224_amd import fp8lin as F

P = 0x100000            # aligned, never dereferenced
NULL = None


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(F.LIB_PATH):
        from paper_2309_17224_amd import build
        build.build()
    return F.lib()


def quant(**kw):
    d = dict(fmt=0, margin=0, bias_pred=None, bias=P, amax_bits=None, flags=None, q=P, ldq=64, qT=None, ldqT=0, ws=P,
             ws_bytes=1 << 30)
    d.update(kw)
    return F.OutQuantise(*[d[n] for n, _ in F.OutQuantise._fields_])


BAD_QUANT = [dict(fmt=9), dict(fmt=-1), dict(margin=1 << 20), dict(bias=None), dict(bias=P + 2), dict(bias_pred=P + 1),
             dict(amax_bits=P + 2), dict(flags=P + 3), dict(q=None), dict(ldq=63), dict(qT=P, ldqT=7), dict(ws=None),
             dict(ws=P + 1), dict(ws_bytes=4)]

FWD_ACT = ("x8 bx w8t bw bias bias_dt act res ldres z ldz y y_dt ldy M N K quant stream").split()
FWD_GLU = ("x8 bx w8t bw bias bias_dt act gu ldgu a lda M N K quant stream").split()
BWD = ("dy8 bg w8 bw z ldz act dz lddz db db_dt M N K quant ws ws_bytes stream").split()
NORM = ("x ldx res ldr dt g b g_dt rows cols eps h ldh y ldy mean rstd quant stream").split()
NORM_BWD = ("dy lddy h ldh dres lddr dt g g_dt mean rstd rows cols dx lddx dg db ws ws_bytes stream").split()
BIAS = ("dy dt rows cols lddy db db_dt ws ws_bytes stream").split()

GOOD = {
    "fp8_linear_fwd_act": (FWD_ACT, dict(x8=P, bx=P, w8t=P, bw=P, bias=P, bias_dt=0, act=2, res=P, ldres=64, z=P, ldz=64,
                                         y=P, y_dt=0, ldy=64, M=8, N=64, K=32, quant=None, stream=None)),
    "fp8_linear_fwd_glu": (FWD_GLU, dict(x8=P, bx=P, w8t=P, bw=P, bias=P, bias_dt=0, act=4, gu=P, ldgu=128, a=P, lda=64,
                                         M=8, N=64, K=32, quant=None, stream=None)),
    "fp8_linear_bwd_dx_act": (BWD, dict(dy8=P, bg=P, w8=P, bw=P, z=P, ldz=64, act=2, dz=P, lddz=64, db=P, db_dt=0, M=8,
                                        N=32, K=64, quant=None, ws=P, ws_bytes=1 << 20, stream=None)),
    "fp8_linear_bwd_dx_glu": (BWD, dict(dy8=P, bg=P, w8=P, bw=P, z=P, ldz=128, act=2, dz=P, lddz=128, db=P, db_dt=0, M=8,
                                        N=32, K=64, quant=None, ws=P, ws_bytes=1 << 20, stream=None)),
    "gpt_layernorm_quantise": (NORM, dict(x=P, ldx=64, res=P, ldr=64, dt=0, g=P, b=P, g_dt=0, rows=8, cols=64, eps=1e-5,
                                          h=P, ldh=64, y=P, ldy=64, mean=P, rstd=P, quant=None, stream=None)),
    "gpt_layernorm_bwd": (NORM_BWD, dict(dy=P, lddy=64, h=P, ldh=64, dres=P, lddr=64, dt=0, g=P, g_dt=0, mean=P, rstd=P,
                                         rows=8, cols=64, dx=P, lddx=64, dg=P, db=P, ws=P, ws_bytes=1 << 20, stream=None)),
    "gpt_bias_grad": (BIAS, dict(dy=P, dt=0, rows=8, cols=64, lddy=64, db=P, db_dt=0, ws=P, ws_bytes=1 << 20,
                                 stream=None)),
}


def call(L, name, **change):
    order, good = GOOD[name]
    assert set(change) <= set(good), change
    d = dict(good, **change)
    if d.get("quant") is not None:
        d["quant"] = ctypes.addressof(d["quant"])
    return getattr(L, name)(*[d[k] for k in order])


COMMON_MM = [dict(M=-1), dict(N=-1), dict(K=-1), dict(M=1 << 41), dict(act=5), dict(act=-1), dict(bw=None), dict(bw=P + 2)]
BAD = {
    "fp8_linear_fwd_act": COMMON_MM + [dict(x8=None), dict(x8=P + 8), dict(w8t=None), dict(w8t=P + 1), dict(bx=None),
                                       dict(y=None), dict(y=P + 1), dict(ldy=63), dict(y_dt=2), dict(y_dt=1, y=P + 2),
                                       dict(bias=P + 1), dict(bias_dt=2), dict(bias_dt=1, bias=P + 2), dict(res=P + 1),
                                       dict(ldres=63), dict(z=P + 1), dict(ldz=63)],
    "fp8_linear_fwd_glu": COMMON_MM + [dict(x8=None), dict(w8t=P + 1), dict(bx=P + 1), dict(a=None), dict(a=P + 1),
                                       dict(lda=63), dict(gu=P + 1), dict(ldgu=127), dict(bias_dt=3)],
    "fp8_linear_bwd_dx_act": COMMON_MM + [dict(dy8=None), dict(w8=P + 4), dict(bg=None), dict(z=None), dict(z=P + 1),
                                          dict(ldz=63), dict(dz=None), dict(lddz=63), dict(db=P + 1), dict(db_dt=2),
                                          dict(ws=None), dict(ws=P + 2), dict(ws_bytes=8)],
    "fp8_linear_bwd_dx_glu": COMMON_MM + [dict(dy8=None), dict(z=None), dict(ldz=127), dict(dz=None), dict(lddz=127),
                                          dict(ws=None), dict(ws_bytes=8)],
    "gpt_layernorm_quantise": [dict(rows=-1), dict(cols=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                               dict(dt=2), dict(g_dt=2), dict(x=None), dict(x=P + 1), dict(ldx=63), dict(y=None),
                               dict(ldy=63), dict(g=None), dict(g=P + 1), dict(b=P + 1), dict(res=P + 1), dict(ldr=63),
                               dict(h=P + 1), dict(ldh=63), dict(mean=P + 2), dict(rstd=P + 1)],
    "gpt_layernorm_bwd": [dict(rows=-1), dict(cols=1 << 41), dict(dt=5), dict(g_dt=5), dict(dy=None), dict(dy=P + 1),
                          dict(lddy=63), dict(h=None), dict(ldh=63), dict(dx=None), dict(lddx=63), dict(dres=P + 1),
                          dict(lddr=63), dict(g=None), dict(mean=None), dict(rstd=None), dict(mean=P + 1), dict(dg=P + 2),
                          dict(db=P + 1), dict(ws=None), dict(ws=P + 2), dict(ws_bytes=8)],
    "gpt_bias_grad": [dict(rows=-1), dict(cols=-1), dict(dt=2), dict(db_dt=2), dict(dy=None), dict(dy=P + 1), dict(lddy=63),
                      dict(db=None), dict(db=P + 1), dict(ws=None), dict(ws=P + 1), dict(ws_bytes=8)],
}


@pytest.mark.parametrize("name", sorted(BAD))
def test_refusals(L, name):
    for change in BAD[name]:
        assert call(L, name, **change) == F.EINVAL, change


@pytest.mark.parametrize("name", [n for n in sorted(GOOD) if "quant" in GOOD[n][0]])
def test_quantise_refusals(L, name):
    glu_bwd = name == "fp8_linear_bwd_dx_glu"
    for bad in BAD_QUANT:
        if name == "gpt_layernorm_quantise" and "qT" in bad:
            continue
        kw = dict(dict(ldq=128) if glu_bwd else {}, **bad)
        if glu_bwd and "ldq" in bad:
            kw["ldq"] = 127
        assert call(L, name, quant=quant(**kw)) == F.EINVAL, bad


def test_unsupported(L):
    assert call(L, "gpt_layernorm_quantise", quant=quant(qT=P, ldqT=8)) == F.ENOTSUP
    assert call(L, "gpt_layernorm_quantise", quant=quant(), dt=1) == F.ENOTSUP
    big = 1 << 31
    assert call(L, "gpt_layernorm_quantise", rows=big) == F.ENOTSUP
    assert call(L, "gpt_layernorm_bwd", rows=big, ws_bytes=1 << 40) == F.ENOTSUP
    assert call(L, "gpt_bias_grad", cols=big, lddy=big, ws_bytes=1 << 60) == F.ENOTSUP
    assert call(L, "fp8_linear_fwd_act", M=big) == F.ENOTSUP
    wide = 1 << 30
    assert call(L, "fp8_linear_fwd_glu", N=wide, lda=wide, ldgu=2 * wide) == F.ENOTSUP
    assert call(L, "fp8_linear_bwd_dx_glu", K=wide, ldz=2 * wide, lddz=2 * wide, db=None) == F.ENOTSUP


def test_more_than_a_launch_counts(L):
    """The last row and column of a tile are 32-bit, and so is the number of a launch's threads."""
    for M in ((1 << 31) - 1, (1 << 31) - 255):
        assert call(L, "fp8_linear_fwd_act", M=M) == F.ENOTSUP
        assert call(L, "fp8_linear_bwd_dx_act", M=M, ws_bytes=1 << 62, db=None) == F.ENOTSUP
    wide = (1 << 31) - 256
    assert call(L, "fp8_linear_fwd_act", N=wide, M=1 << 20, ldy=wide, ldz=wide, ldres=wide) == F.ENOTSUP


def test_a_fused_quantise_without_transposed_codes_refuses_them():
    t = torch.zeros(4, 4, dtype=torch.uint8)
    fq = F.FusedQuant(t, torch.zeros(1, dtype=torch.int32), torch.zeros(8, dtype=torch.uint8), qT=t)
    with pytest.raises(ValueError, match="qT"):
        fq.args()


def test_nothing_to_do_launches_nothing(L):
    """No output and no quantise: OK whatever the pointers."""
    assert call(L, "fp8_linear_fwd_act", M=0, x8=None, y=None) == F.OK
    assert call(L, "fp8_linear_fwd_act", N=0, w8t=None, y=None) == F.OK
    assert call(L, "fp8_linear_fwd_glu", M=0, x8=None, a=None) == F.OK
    assert call(L, "fp8_linear_bwd_dx_act", M=0, dz=None, db=None, ws=None) == F.OK
    assert call(L, "fp8_linear_bwd_dx_glu", K=0, dz=None, ws=None) == F.OK
    assert call(L, "gpt_layernorm_quantise", rows=0, x=None, y=None) == F.OK
    assert call(L, "gpt_layernorm_bwd", rows=0, dx=None, dg=None, db=None) == F.OK
    assert call(L, "gpt_layernorm_bwd", cols=0, dx=None) == F.OK
    assert call(L, "gpt_bias_grad", cols=0, dy=None, db=None) == F.OK


def test_workspace_bytes(L):
    assert L.gpt_layernorm_ws_bytes(0) == 0 and L.gpt_layernorm_ws_bytes(5) == 24
    assert L.gpt_bias_grad_ws_bytes(0, 5) == 0 and L.gpt_bias_grad_ws_bytes(5, 0) == 0
    for rows, cols in ((1, 1), (17, 3), (4096, 5120), (100000, 64)):
        # a row of sums for every 16 rows and the tiles' last ones, at least what gpt_bias_grad's own groups need
        assert L.gpt_bias_grad_ws_bytes(rows, cols) >= 4 * cols * (-(-rows // 16) + 3)
    assert L.gpt_layernorm_bwd_ws_bytes(0, 8) == 0
    assert L.gpt_layernorm_bwd_ws_bytes(1, 8) >= 2 * 8 * 4


def test_binding_refuses_host_tensors():
    u8 = torch.zeros((4, 32), dtype=torch.uint8)
    i = torch.zeros(1, dtype=torch.int32)
    x = torch.zeros((4, 8), dtype=torch.bfloat16)
    s = torch.zeros(4)
    for fn in (lambda: F.fp8_linear_fwd_act(u8, i, u8, i), lambda: F.fp8_linear_fwd_glu(u8, i, u8, i),
               lambda: F.fp8_linear_bwd_dx_act(u8, i, u8, i, x, F.ACT_GELU),
               lambda: F.fp8_linear_bwd_dx_glu(u8, i, u8, i, x), lambda: F.gpt_bias_grad(x),
               lambda: F.gpt_layernorm_quantise(x, x[0]), lambda: F.gpt_layernorm_bwd(x, x, x[0], s, s)):
        with pytest.raises((ValueError, RuntimeError)):
            fn()
