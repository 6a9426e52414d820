"""Thin ctypes binding of libfp8lin.so (include/fp8lin.h).

Argument marshalling only: every function passes device pointers, sizes and
the current HIP stream to the C entry point of the same name and raises
Fp8Error on a non-zero status.  All arithmetic happens in the HIP kernels.
PyTorch provides device memory and streams.  If the shared library has not
been built the first call raises; nothing here falls back to another
implementation.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfp8lin.so")

E4M3, E5M2 = 0, 1
CACHE_BF16 = 16     # format of an unquantised key/value cache
E4_A, E5_A = 2, 3   # the paper's formats (Table 7 rows "(a)"); bias and cast calls only
DT_BF16, DT_F32 = 0, 1
FLAG_NONFINITE, FLAG_ZERO, FLAG_SATURATED = 1, 2, 4
ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = 0, 1, 2, 3, 4
OK, EINVAL, ENOTSUP, EHIP = 0, 1, 2, 3

# Every symbol declared in include/fp8lin.h.
EXPORTS = (
    "fp8_status_string", "fp8_abi_version", "fp8_scale_bias_ws_bytes", "fp8_scale_bias",
    "fp8_bias_from_amax", "fp8_cast_e4", "fp8_cast_e5", "fp8_cast", "fp8_quantise_ws_bytes",
    "fp8_quantise", "fp8_quantise_noalloc", "fp8_quantise_delayed",
    "fp8_quantise_batch",
    "fp8_linear_fwd", "fp8_linear_bwd_dx", "fp8_linear_bias_ws_bytes", "fp8_linear_fwd_bias",
    "fp8_linear_bwd_dx_bias", "fp8_linear_quantise_ws_bytes",
    "fp8_linear_fwd_quantise", "fp8_linear_bwd_dx_quantise",
    "fp8_linear_bwd_dw", "ptq_quantise_weights",
    "fp8_quantise_segments", "fp8_linear_fwd_rows", "fp8_bias_mode",
    "llama_rmsnorm_ws_bytes", "llama_rmsnorm_quantise", "llama_rope_table", "llama_rope",
    "llama_attention_ws_bytes", "llama_attention", "llama_swiglu_ws_bytes", "llama_swiglu_quantise",
    "llama_residual_add",
    "fp8_linear_fwd_act", "fp8_linear_fwd_glu", "fp8_linear_bwd_dx_act", "fp8_linear_bwd_dx_glu",
    "gpt_bias_grad_ws_bytes", "gpt_bias_grad", "gpt_layernorm_ws_bytes", "gpt_layernorm_quantise",
    "gpt_layernorm_bwd_ws_bytes", "gpt_layernorm_bwd",
    "llama_cache_append", "llama_cache_read", "llama_cache_attention_ws_bytes", "llama_cache_attention",
)


class Fp8Error(RuntimeError):
    def __init__(self, fn: str, status: int, msg: str):
        super().__init__(f"{fn} failed with status {status}: {msg}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2309_17224_amd.build` (hipcc, gfx950)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.fp8_status_string.restype = ctypes.c_char_p
        L.fp8_status_string.argtypes = [i32]
        L.fp8_abi_version.restype = i32
        L.fp8_abi_version.argtypes = []
        L.fp8_scale_bias_ws_bytes.restype = sz
        L.fp8_scale_bias_ws_bytes.argtypes = [i64]
        L.fp8_scale_bias.restype = i32
        L.fp8_scale_bias.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp, vp, sz, vp]
        L.fp8_bias_from_amax.restype = i32
        L.fp8_bias_from_amax.argtypes = [vp, i32, i32, vp, vp, vp]
        for name in ("fp8_cast_e4", "fp8_cast_e5"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [vp, i32, i64, i64, i64, vp, vp, i64, vp, i64, vp]
        L.fp8_cast.restype = i32
        L.fp8_cast.argtypes = [vp, i32, i64, i64, i64, i32, vp, vp, i64, vp, i64, vp]
        L.fp8_quantise_ws_bytes.restype = sz
        L.fp8_quantise_ws_bytes.argtypes = [i64, i64]
        L.fp8_quantise.restype = i32
        L.fp8_quantise.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp, i64, vp,
                                   i64, vp, sz, vp]
        L.fp8_quantise_noalloc.restype = i32
        L.fp8_quantise_noalloc.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp, i64, vp,
                                           i64, vp]
        L.fp8_quantise_delayed.restype = i32
        L.fp8_quantise_delayed.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, vp, i64, vp, vp, vp, vp, i64,
                                           vp, i64, vp, sz, vp]
        L.fp8_quantise_batch.argtypes = [i32, vp, i32, i32, i32, vp]
        L.fp8_quantise_batch.restype = i32
        for name in ("fp8_linear_fwd", "fp8_linear_bwd_dx"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, vp, vp]
        L.fp8_linear_bias_ws_bytes.restype = sz
        L.fp8_linear_bias_ws_bytes.argtypes = []
        for name in ("fp8_linear_fwd_bias", "fp8_linear_bwd_dx_bias"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, i32, i32, vp, vp, vp, vp, sz, vp]
        L.fp8_linear_quantise_ws_bytes.restype = sz
        L.fp8_linear_quantise_ws_bytes.argtypes = [i64, i64]
        for name in ("fp8_linear_fwd_quantise", "fp8_linear_bwd_dx_quantise"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, vp, vp, vp, vp, vp, i64, vp,
                          i64, vp, sz, vp]
        L.fp8_linear_bwd_dw.restype = i32
        L.fp8_linear_bwd_dw.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, vp]
        L.fp8_quantise_segments.restype = i32
        L.fp8_quantise_segments.argtypes = [vp, i32, i64, i64, i64, i32, i32, vp, i64, vp, vp, vp, vp, vp, i64,
                                            vp, i64, vp]
        L.fp8_linear_fwd_rows.restype = i32
        L.fp8_linear_fwd_rows.argtypes = [vp, vp, vp, vp, vp, i32, i64, i64, i64, vp, vp]
        L.fp8_bias_mode.restype = i32
        L.fp8_bias_mode.argtypes = [vp, i64, vp, i64, vp, vp]
        f32, f64 = ctypes.c_float, ctypes.c_double
        L.llama_rmsnorm_ws_bytes.restype = sz
        L.llama_rmsnorm_ws_bytes.argtypes = [i64]
        L.llama_rmsnorm_quantise.restype = i32
        L.llama_rmsnorm_quantise.argtypes = [vp, i64, vp, i64, vp, i64, i64, f32, vp, i64, vp, i64, i32, i32,
                                             vp, vp, vp, vp, vp, i64, vp, sz, vp]
        L.llama_rope_table.restype = i32
        L.llama_rope_table.argtypes = [i64, i32, f64, vp, vp]
        L.llama_rope.restype = i32
        L.llama_rope.argtypes = [vp, i64, i64, i32, i32, i64, vp, vp]
        L.llama_attention_ws_bytes.restype = sz
        L.llama_attention_ws_bytes.argtypes = [i64, i64, i32]
        L.llama_attention.restype = i32
        L.llama_attention.argtypes = [vp, i64, i64, i64, i32, i32, i32, vp, i64, i32, i32, vp, vp, vp, vp, vp,
                                      i64, vp, sz, vp]
        L.llama_swiglu_ws_bytes.restype = sz
        L.llama_swiglu_ws_bytes.argtypes = []
        L.llama_swiglu_quantise.restype = i32
        L.llama_swiglu_quantise.argtypes = [vp, i64, i64, i64, vp, i64, i32, i32, vp, vp, vp, vp, vp, i64, vp,
                                            sz, vp]
        L.llama_residual_add.restype = i32
        L.llama_residual_add.argtypes = [vp, vp, vp, i64, vp]
        L.fp8_linear_fwd_act.restype = i32
        L.fp8_linear_fwd_act.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, i64, vp, i64, vp, i32, i64, i64, i64, i64,
                                         vp, vp]
        L.fp8_linear_fwd_glu.restype = i32
        L.fp8_linear_fwd_glu.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, i64, vp, i64, i64, i64, i64, vp, vp]
        for name in ("fp8_linear_bwd_dx_act", "fp8_linear_bwd_dx_glu"):
            f = getattr(L, name)
            f.restype = i32
            f.argtypes = [vp, vp, vp, vp, vp, i64, i32, vp, i64, vp, i32, i64, i64, i64, vp, vp, sz, vp]
        for name in ("gpt_bias_grad_ws_bytes", "gpt_layernorm_bwd_ws_bytes"):
            f = getattr(L, name)
            f.restype = sz
            f.argtypes = [i64, i64]
        L.gpt_bias_grad.restype = i32
        L.gpt_bias_grad.argtypes = [vp, i32, i64, i64, i64, vp, i32, vp, sz, vp]
        L.gpt_layernorm_ws_bytes.restype = sz
        L.gpt_layernorm_ws_bytes.argtypes = [i64]
        L.gpt_layernorm_quantise.restype = i32
        L.gpt_layernorm_quantise.argtypes = [vp, i64, vp, i64, i32, vp, vp, i32, i64, i64, f32, vp, i64, vp, i64, vp, vp,
                                             vp, vp]
        L.gpt_layernorm_bwd.restype = i32
        L.gpt_layernorm_bwd.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, i32, vp, vp, i64, i64, vp, i64, vp, vp, vp,
                                        sz, vp]
        L.llama_cache_append.restype = i32
        L.llama_cache_append.argtypes = [vp, i64, i64, i32, vp, vp, vp, i64, vp, i64, vp]
        L.llama_cache_read.restype = i32
        L.llama_cache_read.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp]
        L.llama_cache_attention_ws_bytes.restype = sz
        L.llama_cache_attention_ws_bytes.argtypes = [i64, i32, vp, vp, i64]
        L.llama_cache_attention.restype = i32
        L.llama_cache_attention.argtypes = [vp, i64, i64, i32, vp, vp, i64, i64, vp, i64, i32, i32, vp, vp, vp, vp,
                                            vp, i64, vp, sz, vp]
        L.ptq_quantise_weights.restype = i32
        L.ptq_quantise_weights.argtypes = [vp, i32, i64, i64, vp, vp, vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def _check(fn: str, status: int) -> None:
    if status != OK:
        raise Fp8Error(fn, status, lib().fp8_status_string(status).decode())


def _p(t: torch.Tensor | None):
    return None if t is None else t.data_ptr()


# The current stream's handle without a Stream object around it, where torch
# offers that (a call of this binding is a few microseconds of host work).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


_BF16 = torch.bfloat16
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return DT_BF16
    if t.dtype == torch.float32:
        return DT_F32
    raise TypeError(f"expected bfloat16 or float32, got {t.dtype}")


def _ld(t: torch.Tensor) -> int:
    """Row stride (elements) of a 2-D tensor whose rows are contiguous."""
    if t.dim() != 2 or (t.stride(1) != 1 and t.size(1) > 1):
        raise ValueError("expected a 2-D tensor with contiguous rows")
    return t.stride(0) if t.size(0) > 1 else max(t.size(1), 1)


def _i32(dev):
    return torch.empty(1, dtype=torch.int32, device=dev)


# ------------------------------------------------------------------ calls
def fp8_scale_bias_ws_bytes(n: int) -> int:
    return int(lib().fp8_scale_bias_ws_bytes(int(n)))


def workspace(n: int, device) -> torch.Tensor:
    return torch.empty(max(fp8_scale_bias_ws_bytes(n), 4), dtype=torch.uint8, device=device)


def fp8_scale_bias(x: torch.Tensor, fmt: int, margin: int = 0, bias=None, amax_bits=None,
                   flags=None, ws=None, stream=None):
    """amax + Eq. 3 bias of a whole tensor.  Returns (bias, amax_bits, flags),
    each a one-element device tensor (int32 / int32 holding uint32 bits)."""
    if not x.is_contiguous():
        raise ValueError("fp8_scale_bias needs a contiguous tensor")
    dev = x.device
    bias = _i32(dev) if bias is None else bias
    amax_bits = _i32(dev) if amax_bits is None else amax_bits
    flags = _i32(dev) if flags is None else flags
    n = x.numel()
    ws = workspace(n, dev) if ws is None else ws
    st = lib().fp8_scale_bias(_p(x), _dt(x), n, fmt, margin, _p(bias), _p(amax_bits), _p(flags),
                              _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check("fp8_scale_bias", st)
    return bias, amax_bits, flags


def fp8_bias_from_amax(amax_bits: torch.Tensor, fmt: int, margin: int = 0, bias=None, flags=None,
                       stream=None):
    dev = amax_bits.device
    bias = _i32(dev) if bias is None else bias
    flags = _i32(dev) if flags is None else flags
    st = lib().fp8_bias_from_amax(_p(amax_bits), fmt, margin, _p(bias), _p(flags), _stream(stream))
    _check("fp8_bias_from_amax", st)
    return bias, flags


def _cast(name: str, x: torch.Tensor, bias: torch.Tensor, q=None, qT=None, want_q=True,
          want_qT=False, stream=None):
    x2 = x if x.dim() == 2 else x.reshape(1, -1)
    rows, cols = x2.shape
    if want_q and q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=x.device)
    st = getattr(lib(), name)(_p(x2), _dt(x2), rows, cols, _ld(x2), _p(bias),
                              _p(q), _ld(q) if q is not None else 0,
                              _p(qT), _ld(qT) if qT is not None else 0, _stream(stream))
    _check(name, st)
    return q, qT


def fp8_cast_e4(x, bias, q=None, qT=None, want_q=True, want_qT=False, stream=None):
    """Scale by 2^bias and cast to E4M3; returns (q, qT)."""
    return _cast("fp8_cast_e4", x, bias, q, qT, want_q, want_qT, stream)


def fp8_cast_e5(x, bias, q=None, qT=None, want_q=True, want_qT=False, stream=None):
    """Scale by 2^bias and cast to E5M2; returns (q, qT)."""
    return _cast("fp8_cast_e5", x, bias, q, qT, want_q, want_qT, stream)


def fp8_cast(x, fmt, bias, q=None, qT=None, want_q=True, want_qT=False, stream=None):
    """Scale by 2^bias and cast to any of E4M3, E5M2, E4_A, E5_A; returns (q, qT)."""
    x2 = x if x.dim() == 2 else x.reshape(1, -1)
    rows, cols = x2.shape
    if want_q and q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=x.device)
    st = lib().fp8_cast(_p(x2), _dt(x2), rows, cols, _ld(x2), fmt, _p(bias),
                        _p(q), _ld(q) if q is not None else 0,
                        _p(qT), _ld(qT) if qT is not None else 0, _stream(stream))
    _check("fp8_cast", st)
    return q, qT


def fp8_quantise_ws_bytes(rows: int, cols: int) -> int:
    return int(lib().fp8_quantise_ws_bytes(rows, cols))


def quantise_workspace(rows: int, cols: int, device) -> torch.Tensor:
    return torch.empty(max(fp8_quantise_ws_bytes(rows, cols), 4), dtype=torch.uint8, device=device)


def fp8_quantise(x: torch.Tensor, fmt: int, margin: int = 0, bias_pred=None, bias=None,
                 amax_bits=None, flags=None, q=None, qT=None, want_q=True, want_qT=False, ws=None,
                 stream=None):
    """amax + Eq. 3 bias + cast of a whole 2-D tensor (codes and/or transposed
    codes).  bias_pred: optional one-element device tensor with a predicted
    bias (may be `bias` itself).  Returns (q, qT, bias, amax_bits, flags)."""
    x2 = x if x.dim() == 2 else x.reshape(1, -1)
    rows, cols = x2.shape
    dev = x.device
    bias = _i32(dev) if bias is None else bias
    amax_bits = _i32(dev) if amax_bits is None else amax_bits
    flags = _i32(dev) if flags is None else flags
    if want_q and q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=dev)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=dev)
    ws = quantise_workspace(rows, cols, dev) if ws is None else ws
    st = lib().fp8_quantise(_p(x2), _dt(x2), rows, cols, _ld(x2), fmt, margin, _p(bias_pred),
                            _p(bias), _p(amax_bits), _p(flags), _p(q),
                            _ld(q) if q is not None else 0, _p(qT),
                            _ld(qT) if qT is not None else 0, _p(ws),
                            ws.numel() * ws.element_size(), _stream(stream))
    _check("fp8_quantise", st)
    return q, qT, bias, amax_bits, flags


def fp8_quantise_delayed(x: torch.Tensor, fmt: int, bias: torch.Tensor, history: torch.Tensor,
                         count: torch.Tensor, margin: int = 0, amax_bits=None, flags=None, q=None, qT=None,
                         want_q=True, want_qT=False, ws=None, stream=None):
    """Delayed scaling: cast with *bias, append amax(x) to the history ring
    and write the next call's bias (Eq. 3 of the history maximum) into bias.
    history: int32 device tensor of history_len words (zeros at first);
    count: one int32 device word.  Returns (q, qT, bias, amax_bits, flags)."""
    x2 = x if x.dim() == 2 else x.reshape(1, -1)
    rows, cols = x2.shape
    dev = x.device
    amax_bits = _i32(dev) if amax_bits is None else amax_bits
    flags = _i32(dev) if flags is None else flags
    if want_q and q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=dev)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=dev)
    ws = quantise_workspace(rows, cols, dev) if ws is None else ws
    st = lib().fp8_quantise_delayed(_p(x2), _dt(x2), rows, cols, _ld(x2), fmt, margin, _p(bias), _p(history),
                                    history.numel(), _p(count), _p(amax_bits), _p(flags), _p(q),
                                    _ld(q) if q is not None else 0, _p(qT), _ld(qT) if qT is not None else 0,
                                    _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check("fp8_quantise_delayed", st)
    return q, qT, bias, amax_bits, flags


NOALLOC_SCRATCH_BYTES = 1048576
NOALLOC_MAX_TILES = 262143


def fp8_quantise_noalloc(x: torch.Tensor, fmt: int, margin: int = 0, bias_pred=None, bias=None,
                         amax_bits=None, flags=None, q=None, qT=None, want_q=True, want_qT=False,
                         stream=None):
    """fp8_quantise with the library's static scratch instead of a workspace
    (nothing allocated by the library; outputs are allocated here only when
    not given).  Returns (q, qT, bias, amax_bits, flags)."""
    x2 = x if x.dim() == 2 else x.reshape(1, -1)
    rows, cols = x2.shape
    dev = x.device
    bias = _i32(dev) if bias is None else bias
    amax_bits = _i32(dev) if amax_bits is None else amax_bits
    flags = _i32(dev) if flags is None else flags
    if want_q and q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=dev)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=dev)
    st = lib().fp8_quantise_noalloc(_p(x2), _dt(x2), rows, cols, _ld(x2), fmt, margin, _p(bias_pred),
                                    _p(bias), _p(amax_bits), _p(flags), _p(q),
                                    _ld(q) if q is not None else 0, _p(qT),
                                    _ld(qT) if qT is not None else 0, _stream(stream))
    _check("fp8_quantise_noalloc", st)
    return q, qT, bias, amax_bits, flags


class QuantiseArgs(ctypes.Structure):
    """fp8_quantise_args of the C header (device pointers, sizes)."""
    _fields_ = [("x", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ldx", ctypes.c_int64), ("bias_pred", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("amax_bits", ctypes.c_void_p), ("flags", ctypes.c_void_p), ("q", ctypes.c_void_p),
                ("ldq", ctypes.c_int64), ("qT", ctypes.c_void_p), ("ldqT", ctypes.c_int64),
                ("ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t)]


QUANTISE_BATCH_MAX = 4


def fp8_quantise_batch(items, fmt: int, margin: int = 0, stream=None):
    """fp8_quantise of several 2-D tensors of one dtype in two launches (same
    bits as separate calls).  items: dicts with x, bias, ws and optionally
    bias_pred, amax_bits, flags, q, qT (outputs are not allocated here)."""
    arr = (QuantiseArgs * max(len(items), 1))()
    dt = _dt(items[0]["x"]) if items else DT_BF16
    for a, it in zip(arr, items):
        x = it["x"]
        q, qT, ws = it.get("q"), it.get("qT"), it["ws"]
        a.x, a.rows, a.cols, a.ldx = _p(x), x.shape[0], x.shape[1], _ld(x)
        a.bias_pred, a.bias = _p(it.get("bias_pred")), _p(it["bias"])
        a.amax_bits, a.flags = _p(it.get("amax_bits")), _p(it.get("flags"))
        a.q, a.ldq = _p(q), _ld(q) if q is not None else 0
        a.qT, a.ldqT = _p(qT), _ld(qT) if qT is not None else 0
        a.ws, a.ws_bytes = _p(ws), ws.numel() * ws.element_size()
    st = lib().fp8_quantise_batch(len(items), ctypes.cast(arr, ctypes.c_void_p), dt, fmt, margin,
                                  _stream(stream))
    _check("fp8_quantise_batch", st)


def _out(shape, out_dt, dev, out):
    if out is not None:
        return out
    return torch.empty(shape, dtype=torch.bfloat16 if out_dt == DT_BF16 else torch.float32,
                       device=dev)


def _odt(out_dt: int, out) -> int:
    return out_dt if out is None else _dt(out)


def fp8_linear_fwd(x8, bx, w8t, bw, out_dt=DT_BF16, y=None, y_amax_bits=None, stream=None):
    """Y [M,N] = 2^-(bx+bw) X8 [M,K] . W8T [N,K]^T."""
    M, K = x8.shape
    N = w8t.shape[0]
    y = _out((M, N), out_dt, x8.device, y)
    st = lib().fp8_linear_fwd(_p(x8), _p(bx), _p(w8t), _p(bw), _p(y), _odt(out_dt, y), M, N, K,
                              _p(y_amax_bits), _stream(stream))
    _check("fp8_linear_fwd", st)
    return y


def fp8_linear_bwd_dx(dy8, bg, w8, bw, out_dt=DT_BF16, dx=None, dx_amax_bits=None, stream=None):
    """dX [M,K] = 2^-(bg+bw) dY8 [M,N] . W8 [K,N]^T."""
    M, N = dy8.shape
    K = w8.shape[0]
    dx = _out((M, K), out_dt, dy8.device, dx)
    st = lib().fp8_linear_bwd_dx(_p(dy8), _p(bg), _p(w8), _p(bw), _p(dx), _odt(out_dt, dx), M, N, K,
                                 _p(dx_amax_bits), _stream(stream))
    _check("fp8_linear_bwd_dx", st)
    return dx


def bias_workspace(device) -> torch.Tensor:
    """Workspace of fp8_linear_fwd_bias / fp8_linear_bwd_dx_bias: zeros, and
    left zero by every completed call (one per stream of concurrent calls)."""
    return torch.zeros(int(lib().fp8_linear_bias_ws_bytes()) // 4, dtype=torch.int32, device=device)


def _gemm_bias(name, a8, ba, b8, bb, out, out_dt, rows, cols, kc, fmt, margin, bias, amax_bits, flags,
               ws, stream):
    dev = a8.device
    out = _out((rows, cols), out_dt, dev, out)
    bias = _i32(dev) if bias is None else bias
    amax_bits = _i32(dev) if amax_bits is None else amax_bits
    flags = _i32(dev) if flags is None else flags
    ws = bias_workspace(dev) if ws is None else ws
    st = getattr(lib(), name)(_p(a8), _p(ba), _p(b8), _p(bb), _p(out), _odt(out_dt, out), *(
        (rows, cols, kc) if name == "fp8_linear_fwd_bias" else (rows, kc, cols)),
        fmt, margin, _p(bias), _p(amax_bits), _p(flags), _p(ws), ws.numel() * ws.element_size(),
        _stream(stream))
    _check(name, st)
    return out, bias, amax_bits, flags


def fp8_linear_fwd_bias(x8, bx, w8t, bw, fmt=E4M3, margin=0, out_dt=DT_BF16, y=None, bias=None,
                        amax_bits=None, flags=None, ws=None, stream=None):
    """Y = fp8_linear_fwd(...) with the Eq. 3 bias of Y (format fmt) from the
    same launch.  Returns (y, bias, amax_bits, flags)."""
    M, K = x8.shape
    N = w8t.shape[0]
    return _gemm_bias("fp8_linear_fwd_bias", x8, bx, w8t, bw, y, out_dt, M, N, K, fmt, margin, bias,
                      amax_bits, flags, ws, stream)


def fp8_linear_bwd_dx_bias(dy8, bg, w8, bw, fmt=E5M2, margin=0, out_dt=DT_BF16, dx=None, bias=None,
                           amax_bits=None, flags=None, ws=None, stream=None):
    """dX = fp8_linear_bwd_dx(...) with the Eq. 3 bias of dX from the same
    launch.  Returns (dx, bias, amax_bits, flags)."""
    M, N = dy8.shape
    K = w8.shape[0]
    return _gemm_bias("fp8_linear_bwd_dx_bias", dy8, bg, w8, bw, dx, out_dt, M, K, N, fmt, margin, bias,
                      amax_bits, flags, ws, stream)


def _gemm_quantise(name, a8, ba, b8, bb, out, rows, cols, kc, fmt, margin, bias_pred, bias,
                   amax_bits, flags, q, qT, want_qT, ws, stream):
    dev = a8.device
    out = _out((rows, cols), DT_BF16, dev, out)
    bias = _i32(dev) if bias is None else bias
    amax_bits = _i32(dev) if amax_bits is None else amax_bits
    flags = _i32(dev) if flags is None else flags
    if q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=dev)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=dev)
    if ws is None:
        ws = torch.empty(max(int(lib().fp8_linear_quantise_ws_bytes(rows, cols)), 4), dtype=torch.uint8,
                         device=dev)
    st = getattr(lib(), name)(_p(a8), _p(ba), _p(b8), _p(bb), _p(out), *(
        (rows, cols, kc) if name == "fp8_linear_fwd_quantise" else (rows, kc, cols)),
        fmt, margin, _p(bias_pred), _p(bias), _p(amax_bits), _p(flags), _p(q), _ld(q), _p(qT),
        _ld(qT) if qT is not None else 0, _p(ws), ws.numel() * ws.element_size(), _stream(stream))
    _check(name, st)
    return out, q, qT, bias, amax_bits, flags


def fp8_linear_fwd_quantise(x8, bx, w8t, bw, fmt=E4M3, margin=0, bias_pred=None, y=None, bias=None,
                            amax_bits=None, flags=None, y8=None, y8t=None, want_y8t=False, ws=None,
                            stream=None):
    """Y = fp8_linear_fwd(...) (bf16) and its FP8 codes, bias, amax, flags from
    the epilogue.  Returns (y, y8, y8t, bias, amax_bits, flags)."""
    M, K = x8.shape
    N = w8t.shape[0]
    return _gemm_quantise("fp8_linear_fwd_quantise", x8, bx, w8t, bw, y, M, N, K, fmt, margin,
                          bias_pred, bias, amax_bits, flags, y8, y8t, want_y8t, ws, stream)


def fp8_linear_bwd_dx_quantise(dy8, bg, w8, bw, fmt=E5M2, margin=0, bias_pred=None, dx=None,
                               bias=None, amax_bits=None, flags=None, dx8=None, dx8t=None,
                               want_dx8t=False, ws=None, stream=None):
    """dX = fp8_linear_bwd_dx(...) (bf16) and its FP8 codes etc.  Returns
    (dx, dx8, dx8t, bias, amax_bits, flags)."""
    M, N = dy8.shape
    K = w8.shape[0]
    return _gemm_quantise("fp8_linear_bwd_dx_quantise", dy8, bg, w8, bw, dx, M, K, N, fmt, margin,
                          bias_pred, bias, amax_bits, flags, dx8, dx8t, want_dx8t, ws, stream)


def fp8_linear_bwd_dw(x8t, bx, dy8t, bg, out_dt=DT_F32, dw=None, stream=None):
    """dW [K,N] = 2^-(bx+bg) X8T [K,M] . dY8T [N,M]^T."""
    K, M = x8t.shape
    N = dy8t.shape[0]
    dw = _out((K, N), out_dt, x8t.device, dw)
    st = lib().fp8_linear_bwd_dw(_p(x8t), _p(bx), _p(dy8t), _p(bg), _p(dw), _odt(out_dt, dw), M, N, K,
                                 _stream(stream))
    _check("fp8_linear_bwd_dw", st)
    return dw


def ptq_quantise_weights(w, want_w8=True, want_w8t=True, w8=None, w8t=None, bw=None, flags=None,
                         ws=None, stream=None):
    """Post-training quantisation of a [K, N] weight: returns (w8, w8t, bw, flags)."""
    if not w.is_contiguous():
        raise ValueError("ptq_quantise_weights needs a contiguous weight")
    K, N = w.shape
    dev = w.device
    if want_w8 and w8 is None:
        w8 = torch.empty((K, N), dtype=torch.uint8, device=dev)
    if want_w8t and w8t is None:
        w8t = torch.empty((N, K), dtype=torch.uint8, device=dev)
    bw = _i32(dev) if bw is None else bw
    flags = _i32(dev) if flags is None else flags
    ws = workspace(K * N, dev) if ws is None else ws
    st = lib().ptq_quantise_weights(_p(w), _dt(w), K, N, _p(w8), _p(w8t), _p(bw), _p(flags), _p(ws),
                                    ws.numel() * ws.element_size(), _stream(stream))
    _check("ptq_quantise_weights", st)
    return w8, w8t, bw, flags


def fp8_quantise_segments(x: torch.Tensor, offsets: torch.Tensor, fmt: int, margin: int = 0, bias=None,
                          amax_bits=None, flags=None, row_bias=None, q=None, qT=None, want_q=True,
                          want_qT=False, stream=None):
    """amax + Eq. 3 bias + cast per row segment (rows offsets[s] .. offsets[s+1]-1,
    offsets a device int32 [nseg + 1]).  Returns (q, qT, bias[nseg],
    amax_bits[nseg], flags[nseg], row_bias[rows])."""
    rows, cols = x.shape
    dev = x.device
    nseg = offsets.numel() - 1
    i32 = dict(dtype=torch.int32, device=dev)
    bias = torch.empty(nseg, **i32) if bias is None else bias
    amax_bits = torch.empty(nseg, **i32) if amax_bits is None else amax_bits
    flags = torch.empty(nseg, **i32) if flags is None else flags
    row_bias = torch.empty(max(rows, 1), **i32) if row_bias is None else row_bias
    if want_q and q is None:
        q = torch.empty((rows, cols), dtype=torch.uint8, device=dev)
    if want_qT and qT is None:
        qT = torch.empty((cols, rows), dtype=torch.uint8, device=dev)
    st = lib().fp8_quantise_segments(_p(x), _dt(x), rows, cols, _ld(x), fmt, margin, _p(offsets), nseg,
                                     _p(bias), _p(amax_bits), _p(flags), _p(row_bias), _p(q),
                                     _ld(q) if q is not None else 0, _p(qT), _ld(qT) if qT is not None else 0,
                                     _stream(stream))
    _check("fp8_quantise_segments", st)
    return q, qT, bias, amax_bits, flags, row_bias[:rows]


def fp8_linear_fwd_rows(x8, bx_rows, w8t, bw, out_dt=DT_BF16, y=None, y_amax_bits=None, stream=None):
    """Y [M,N] = 2^-(bx_rows[m]+bw) X8 [M,K] . W8T [N,K]^T (one activation bias per row)."""
    M, K = x8.shape
    N = w8t.shape[0]
    y = _out((M, N), out_dt, x8.device, y)
    st = lib().fp8_linear_fwd_rows(_p(x8), _p(bx_rows), _p(w8t), _p(bw), _p(y), _odt(out_dt, y), M, N, K,
                                   _p(y_amax_bits), _stream(stream))
    _check("fp8_linear_fwd_rows", st)
    return y


def fp8_bias_mode(bias: torch.Tensor, ring: torch.Tensor, count: torch.Tensor, stream=None):
    """Append the mode of `bias` to the device ring buffer `ring` at
    count % capacity and increment `count` (one-element int32), on the device."""
    st = lib().fp8_bias_mode(_p(bias), bias.numel(), _p(ring), ring.numel(), _p(count), _stream(stream))
    _check("fp8_bias_mode", st)


# ------------------------------------------------------------------ decoder-layer glue
class FusedQuant:
    """Arguments of a quantise fused into a glue call: codes q [rows, cols]
    (uint8), the format and margin, an optional predicted bias, and one-element
    int32 device tensors for the bias, amax bits and flags; ws is the op's
    workspace (uint8 tensor).  qT: the transposed codes [cols, rows], for the
    calls that write them (the matmuls of the feed-forward block)."""

    def __init__(self, q, bias, ws, fmt=E4M3, margin=0, bias_pred=None, amax_bits=None, flags=None, qT=None):
        self.q, self.bias, self.ws = q, bias, ws
        self.fmt, self.margin, self.bias_pred = fmt, margin, bias_pred
        self.amax_bits, self.flags, self.qT = amax_bits, flags, qT

    def args(self):
        if self.qT is not None:
            raise ValueError("fq.qT: this call writes no transposed codes")
        return (self.fmt, self.margin, _p(self.bias_pred), _p(self.bias), _p(self.amax_bits), _p(self.flags),
                _p(self.q), _ld(self.q), _p(self.ws), self.ws.numel() * self.ws.element_size())


_NO_QUANT = (E4M3, 0, None, None, None, None, None, 0, None, 0)


def _bf16(t: torch.Tensor, name: str) -> None:
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name}: expected bfloat16, got {t.dtype}")


def llama_rmsnorm_ws_bytes(rows: int) -> int:
    return int(lib().llama_rmsnorm_ws_bytes(int(rows)))


def llama_rmsnorm_quantise(x, g, eps=1e-5, res=None, h=None, y=None, fq: FusedQuant | None = None, stream=None):
    """y = RMSNorm(x [+ res]) * g (and h = x + res), optionally with the fused
    quantise of y.  Returns y."""
    _bf16(x, "x")
    rows, cols = x.shape
    y = torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device) if y is None else y
    st = lib().llama_rmsnorm_quantise(_p(x), _ld(x), _p(res), _ld(res) if res is not None else 0, _p(g), rows,
                                      cols, float(eps), _p(h), _ld(h) if h is not None else 0, _p(y), _ld(y),
                                      *(fq.args() if fq else _NO_QUANT), _stream(stream))
    _check("llama_rmsnorm_quantise", st)
    return y


def llama_rope_table(seq_len: int, d_head: int, theta: float = 10000.0, table=None, device=None, stream=None):
    if table is None:
        table = torch.empty(seq_len * d_head, dtype=torch.float32, device=device)
    st = lib().llama_rope_table(int(seq_len), int(d_head), float(theta), _p(table), _stream(stream))
    _check("llama_rope_table", st)
    return table


def llama_rope(x, n_heads: int, d_head: int, seq_len: int, table, stream=None):
    """Rotary embedding in place on the first n_heads heads of x (a 2-D view
    whose rows are contiguous, e.g. the Q and K columns of the QKV output)."""
    _bf16(x, "x")
    rows = x.shape[0]
    ld = x.stride(0)
    st = lib().llama_rope(_p(x), rows, ld, int(n_heads), int(d_head), int(seq_len), _p(table), _stream(stream))
    _check("llama_rope", st)
    return x


def llama_attention_ws_bytes(rows: int, seq_len: int, n_heads: int) -> int:
    return int(lib().llama_attention_ws_bytes(int(rows), int(seq_len), int(n_heads)))


def llama_attention(qkv, seq_len: int, n_heads: int, n_kv_heads: int, d_head: int = 128, o=None,
                    fq: FusedQuant | None = None, stream=None):
    """Causal grouped-query attention over the QKV output; returns o."""
    _bf16(qkv, "qkv")
    rows = qkv.shape[0]
    o = torch.empty((rows, n_heads * d_head), dtype=torch.bfloat16, device=qkv.device) if o is None else o
    st = lib().llama_attention(_p(qkv), rows, _ld(qkv), int(seq_len), int(n_heads), int(n_kv_heads), int(d_head),
                               _p(o), _ld(o), *(fq.args() if fq else _NO_QUANT), _stream(stream))
    _check("llama_attention", st)
    return o


def llama_swiglu_ws_bytes() -> int:
    return int(lib().llama_swiglu_ws_bytes())


def llama_swiglu_quantise(gu, ffn: int, a=None, fq: FusedQuant | None = None, stream=None):
    """a = silu(gate) * up over the fused gate+up output; returns a."""
    _bf16(gu, "gu")
    rows = gu.shape[0]
    a = torch.empty((rows, ffn), dtype=torch.bfloat16, device=gu.device) if a is None else a
    st = lib().llama_swiglu_quantise(_p(gu), _ld(gu), rows, int(ffn), _p(a), _ld(a),
                                     *(fq.args() if fq else _NO_QUANT), _stream(stream))
    _check("llama_swiglu_quantise", st)
    return a


def llama_residual_add(a, b, out=None, stream=None):
    _bf16(a, "a")
    out = torch.empty_like(a) if out is None else out
    st = lib().llama_residual_add(_p(a), _p(b), _p(out), a.numel(), _stream(stream))
    _check("llama_residual_add", st)
    return out


# ------------------------------------------------------------------ the feed-forward block
class OutQuantise(ctypes.Structure):
    """fp8_out_quantise of the C header."""
    _fields_ = [("fmt", ctypes.c_int32), ("margin", ctypes.c_int32), ("bias_pred", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("amax_bits", ctypes.c_void_p), ("flags", ctypes.c_void_p),
                ("q", ctypes.c_void_p), ("ldq", ctypes.c_int64), ("qT", ctypes.c_void_p), ("ldqT", ctypes.c_int64),
                ("ws", ctypes.c_void_p), ("ws_bytes", ctypes.c_size_t)]


# (A call of these is a few microseconds of host work, as long as its kernel where the
# tensors are small: what is right is looked at once, what is wrong is named apart.)
def _gpu(t: torch.Tensor, name: str) -> int:
    """The GPU of a call's first operand: the current one, whose stream runs the call."""
    dev = t.get_device()
    if dev < 0 or _current() != dev:
        raise ValueError(f"{name}: on {t.device}, which is not the current GPU")
    return dev


def _rows(t: torch.Tensor, name: str, rows: int, cols: int, dev: int, dtype=_BF16) -> int:
    """Row stride of a tensor [rows, cols] of a type with contiguous rows, on GPU dev."""
    if t.dtype is dtype and t.shape == (rows, cols) and t.get_device() == dev:
        if t.is_contiguous():
            return cols or 1
        ld, one = t.stride()
        if (one == 1 or cols <= 1) and (ld >= cols or rows <= 1):
            return ld if rows > 1 else cols or 1
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name}: on {t.device}, the call on GPU {dev}")
    raise ValueError(f"{name}: expected [{rows}, {cols}] with contiguous rows that do not overlap, "
                     f"got {tuple(t.shape)}, strides {t.stride()}")


def _vec(t: torch.Tensor, name: str, n: int, dev: int, dtypes) -> int:
    """Address of a contiguous vector of n elements (any shape) of one of the types on GPU dev."""
    if t.dtype in dtypes and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: expected one of {dtypes}, got {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name}: on {t.device}, the call on GPU {dev}")
    raise ValueError(f"{name}: expected {n} contiguous elements, got {tuple(t.shape)}, strides {t.stride()}")


def _float(t: torch.Tensor, name: str) -> torch.dtype:
    dt = t.dtype
    if dt is not _BF16 and dt is not torch.float32:
        raise TypeError(f"{name}: expected torch.bfloat16 or torch.float32, got {dt}")
    return dt


def _stream_on(stream, dev: int):
    """The stream of a call on GPU dev, the current one."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(dev)
    if stream is not None and stream.device_index != dev:
        raise ValueError(f"stream: of GPU {stream.device_index}, the call on GPU {dev}")
    return _stream(stream)


_FLOATS = (torch.bfloat16, torch.float32)
_F32 = (torch.float32,)
_INT = (torch.int32,)
_U8 = (torch.uint8,)


def _made(shape, dtype, device, stream) -> torch.Tensor:
    """A tensor of the memory of the stream that a call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _scratch(ws, nbytes: int, dev: int, device, stream):
    """Address and bytes of a workspace; made for the call where none is given."""
    if ws is None:
        ws = _made(max(nbytes, 4), torch.uint8, device, stream)
    elif ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"ws: expected a contiguous tensor on GPU {dev}")
    return ws.data_ptr(), ws.nbytes


def _out_quantise(fq: FusedQuant | None, rows: int, cols: int, dev: int):
    """fp8_out_quantise of a FusedQuant (kept alive by the caller until the call has returned)."""
    if fq is None:
        return None
    ldq = _rows(fq.q, "fq.q", rows, cols, dev, torch.uint8)
    qT, ldqT = None, 0
    if fq.qT is not None:
        qT, ldqT = fq.qT.data_ptr(), _rows(fq.qT, "fq.qT", cols, rows, dev, torch.uint8)
    one = [None if t is None else _vec(t, "fq's bias, prediction, amax and flags", 1, dev, _INT)
           for t in (fq.bias_pred, fq.bias, fq.amax_bits, fq.flags)]
    ws, nws = _scratch(fq.ws, 0, dev, None, None)
    return OutQuantise(fq.fmt, fq.margin, *one, fq.q.data_ptr(), ldq, qT, ldqT, ws, nws)


def _ref(quant):
    return None if quant is None else ctypes.addressof(quant)


def _operands(a8, ba, b8, bb, names):
    """Checks of a matmul's operands [M, K] and [N, K] and their biases: their addresses, M, N, K and
    the GPU."""
    dev = _gpu(a8, names[0])
    u8, i32 = torch.uint8, torch.int32
    if a8.dtype is u8 and b8.dtype is u8 and ba.dtype is i32 and bb.dtype is i32:
        sa, sb = a8.shape, b8.shape
        if (len(sa) == 2 and len(sb) == 2 and sa[1] == sb[1] and a8.is_contiguous() and b8.is_contiguous()
                and ba.numel() == 1 and bb.numel() == 1 and b8.get_device() == dev and ba.get_device() == dev
                and bb.get_device() == dev):
            return (a8.data_ptr(), ba.data_ptr(), b8.data_ptr(), bb.data_ptr()), sa[0], sb[0], sa[1], dev
    if a8.dim() != 2 or b8.dim() != 2 or a8.shape[1] != b8.shape[1]:
        raise ValueError(f"{names[0]}, {names[2]}: expected [M, K] and [N, K], got {tuple(a8.shape)} and {tuple(b8.shape)}")
    for t, name, n, kind in ((a8, names[0], a8.numel(), _U8), (ba, names[1], 1, _INT), (b8, names[2], b8.numel(), _U8),
                             (bb, names[3], 1, _INT)):
        _vec(t, name, n, dev, kind)
    raise ValueError(f"{names}: unusable operands")


_FWD_NAMES = ("x8", "bx", "w8t", "bw")
_BWD_NAMES = ("dy8", "bg", "w8", "bw")


def fp8_linear_quantise_ws_bytes(rows: int, cols: int) -> int:
    return int(lib().fp8_linear_quantise_ws_bytes(int(rows), int(cols)))


def fp8_linear_fwd_act(x8, bx, w8t, bw, act: int = ACT_NONE, bias=None, res=None, z=None, out_dt: int = DT_BF16, y=None,
                       fq: FusedQuant | None = None, stream=None):
    """y = act(z) + res, z = 2^-(bx+bw) X8 [M,K] . W8T [N,K]^T + bias, in one matmul.
    bias: [N], bf16 or fp32.  res: [M, N] of y's type (may be y).  z: bf16 [M, N], written
    for fp8_linear_bwd_dx_act.  fq: codes of y (ws of fp8_linear_quantise_ws_bytes(M, N)
    bytes).  Returns y."""
    ops, M, N, K, dev = _operands(x8, bx, w8t, bw, _FWD_NAMES)
    if y is None:
        y = _made((M, N), torch.bfloat16 if out_dt == DT_BF16 else torch.float32, x8.device, stream)
    dt = _float(y, "y")
    ldy = _rows(y, "y", M, N, dev, dt)
    b, b_dt = (None, 0) if bias is None else (_vec(bias, "bias", N, dev, _FLOATS), _dt(bias))
    r, ldr = (None, 0) if res is None else (res.data_ptr(), _rows(res, "res", M, N, dev, dt))
    zp, ldz = (None, 0) if z is None else (z.data_ptr(), _rows(z, "z", M, N, dev))
    quant = None if fq is None else _out_quantise(fq, M, N, dev)
    st = lib().fp8_linear_fwd_act(*ops, b, b_dt, act, r, ldr, zp, ldz, y.data_ptr(), DT_BF16 if dt is _BF16 else DT_F32,
                                  ldy, M, N, K, _ref(quant), _stream_on(stream, dev))
    if st:
        _check("fp8_linear_fwd_act", st)
    return y


def fp8_linear_fwd_glu(x8, bx, w8t, bw, act: int = ACT_SILU, bias=None, gu=None, a=None, fq: FusedQuant | None = None,
                       stream=None):
    """a = act(g) * u, (g | u) = 2^-(bx+bw) X8 [M,K] . W8T [2N,K]^T + bias (gate rows of W8T
    first), in one matmul.  bias: [2 N].  gu: bf16 [M, 2 N], written for
    fp8_linear_bwd_dx_glu.  fq: codes of a [M, N].  Returns a."""
    ops, M, N2, K, dev = _operands(x8, bx, w8t, bw, _FWD_NAMES)
    if N2 % 2:
        raise ValueError(f"w8t: expected as many gate rows as up rows, got {N2} rows")
    N = N2 // 2
    if a is None:
        a = _made((M, N), torch.bfloat16, x8.device, stream)
    lda = _rows(a, "a", M, N, dev)
    b, b_dt = (None, 0) if bias is None else (_vec(bias, "bias", N2, dev, _FLOATS), _dt(bias))
    g, ldgu = (None, 0) if gu is None else (gu.data_ptr(), _rows(gu, "gu", M, N2, dev))
    quant = None if fq is None else _out_quantise(fq, M, N, dev)
    st = lib().fp8_linear_fwd_glu(*ops, b, b_dt, act, g, ldgu, a.data_ptr(), lda, M, N, K, _ref(quant),
                                  _stream_on(stream, dev))
    if st:
        _check("fp8_linear_fwd_glu", st)
    return a


def gpt_bias_grad_ws_bytes(rows: int, cols: int) -> int:
    return int(lib().gpt_bias_grad_ws_bytes(int(rows), int(cols)))


def bias_grad_workspace(rows: int, cols: int, device) -> torch.Tensor:
    """Workspace of gpt_bias_grad, and of the backward matmuls' bias gradients
    (rows and columns of their output)."""
    return torch.empty(max(gpt_bias_grad_ws_bytes(rows, cols), 4), dtype=torch.uint8, device=device)


def _linear_bwd(name, dy8, bg, w8, bw, saved, saved_name, act, out, out_name, wide, db, fq, ws, stream):
    ops, M, K, N, dev = _operands(dy8, bg, w8, bw, _BWD_NAMES)  # [M, N] and [K, N]
    cols = wide * K
    lds = _rows(saved, saved_name, M, cols, dev)
    if out is None:
        out = _made((M, cols), torch.bfloat16, dy8.device, stream)
    ldo = _rows(out, out_name, M, cols, dev)
    quant = None if fq is None else _out_quantise(fq, M, cols, dev)
    d, d_dt, w = None, 0, (None, 0)
    if db is not None:
        d, d_dt = _vec(db, "db", cols, dev, _FLOATS), _dt(db)
        w = _scratch(ws, gpt_bias_grad_ws_bytes(M, cols) if ws is None else 0, dev, dy8.device, stream)
    st = getattr(lib(), name)(*ops, saved.data_ptr(), lds, act, out.data_ptr(), ldo, d, d_dt, M, N, K, _ref(quant), *w,
                              _stream_on(stream, dev))
    if st:
        _check(name, st)
    return out


def fp8_linear_bwd_dx_act(dy8, bg, w8, bw, z, act: int, dz=None, db=None, fq: FusedQuant | None = None, ws=None,
                          stream=None):
    """dz = t act'(z), t = 2^-(bg+bw) dY8 [M,N] . W8 [K,N]^T: the gradient that reaches the
    linear before, whose output before its activation was z [M, K].  db: its bias gradient
    [K] (bf16 or fp32), the sum of t act'(z) over rows, with ws of gpt_bias_grad_ws_bytes(M,
    K) bytes.  fq: codes of dz.  dz may be z.  Returns dz."""
    return _linear_bwd("fp8_linear_bwd_dx_act", dy8, bg, w8, bw, z, "z", act, dz, "dz", 1, db, fq, ws, stream)


def fp8_linear_bwd_dx_glu(dy8, bg, w8, bw, gu, act: int = ACT_SILU, dgu=None, db=None, fq: FusedQuant | None = None,
                          ws=None, stream=None):
    """dg = t u act'(g) and du = t act(g), t = 2^-(bg+bw) dY8 [M,N] . W8 [K,N]^T: the gradients
    of the gate's and the up projection's outputs gu [M, 2 K], side by side.  db: their sums
    over rows [2 K].  fq: codes of dgu.  dgu may be gu.  Returns dgu."""
    return _linear_bwd("fp8_linear_bwd_dx_glu", dy8, bg, w8, bw, gu, "gu", act, dgu, "dgu", 2, db, fq, ws, stream)


def gpt_bias_grad(dy, db=None, ws=None, stream=None):
    """Sum over the rows of dy [rows, cols] (bf16 or fp32).  db: [cols], bf16 or fp32 (fp32
    where it is made here).  Returns db."""
    dev = _gpu(dy, "dy")
    rows, cols = dy.shape
    ld = _rows(dy, "dy", rows, cols, dev, _float(dy, "dy"))
    if db is None:
        db = _made((cols,), torch.float32, dy.device, stream)
    d = _vec(db, "db", cols, dev, _FLOATS)
    w = _scratch(ws, gpt_bias_grad_ws_bytes(rows, cols) if ws is None else 0, dev, dy.device, stream)
    st = lib().gpt_bias_grad(dy.data_ptr(), _dt(dy), rows, cols, ld, d, _dt(db), *w, _stream_on(stream, dev))
    if st:
        _check("gpt_bias_grad", st)
    return db


def gpt_layernorm_ws_bytes(rows: int) -> int:
    return int(lib().gpt_layernorm_ws_bytes(int(rows)))


def gpt_layernorm_quantise(x, g, b=None, eps=1e-5, res=None, h=None, y=None, mean=None, rstd=None,
                           fq: FusedQuant | None = None, stream=None):
    """y = LayerNorm(h) * g + b, h = x [+ res] (bf16 or fp32; g and b of one type).  h, mean,
    rstd: written where given (mean and rstd fp32 [rows], for gpt_layernorm_bwd).  fq: codes
    of a bf16 y, ws of gpt_layernorm_ws_bytes(rows) bytes, no qT.  Returns y."""
    dev = _gpu(x, "x")
    rows, cols = x.shape
    dt = _float(x, "x")
    ldx = _rows(x, "x", rows, cols, dev, dt)
    if y is None:
        y = _made((rows, cols), dt, x.device, stream)
    ldy = _rows(y, "y", rows, cols, dev, dt)
    r, ldr = (None, 0) if res is None else (res.data_ptr(), _rows(res, "res", rows, cols, dev, dt))
    hp, ldh = (None, 0) if h is None else (h.data_ptr(), _rows(h, "h", rows, cols, dev, dt))
    gp = _vec(g, "g", cols, dev, _FLOATS)
    bp = None if b is None else _vec(b, "b", cols, dev, (g.dtype,))
    mp = None if mean is None else _vec(mean, "mean", rows, dev, _F32)
    sp = None if rstd is None else _vec(rstd, "rstd", rows, dev, _F32)
    quant = None if fq is None else _out_quantise(fq, rows, cols, dev)
    st = lib().gpt_layernorm_quantise(x.data_ptr(), ldx, r, ldr, DT_BF16 if dt is _BF16 else DT_F32, gp, bp, _dt(g), rows,
                                      cols, eps, hp, ldh, y.data_ptr(), ldy, mp, sp, _ref(quant), _stream_on(stream, dev))
    if st:
        _check("gpt_layernorm_quantise", st)
    return y


def gpt_layernorm_bwd_ws_bytes(rows: int, cols: int) -> int:
    return int(lib().gpt_layernorm_bwd_ws_bytes(int(rows), int(cols)))


def layernorm_bwd_workspace(rows: int, cols: int, device) -> torch.Tensor:
    return torch.empty(max(gpt_layernorm_bwd_ws_bytes(rows, cols), 4), dtype=torch.uint8, device=device)


def gpt_layernorm_bwd(dy, h, g, mean, rstd, dres=None, dx=None, dg=None, db=None, want_params=True, ws=None, stream=None):
    """Gradients of gpt_layernorm_quantise: dx (with dres, the gradient that reaches h past the
    norm, added), dg and db (fp32 [cols]; made here with want_params).  h: what was
    normalised.  Returns (dx, dg, db)."""
    dev = _gpu(dy, "dy")
    rows, cols = dy.shape
    dt = _float(dy, "dy")
    lddy = _rows(dy, "dy", rows, cols, dev, dt)
    ldh = _rows(h, "h", rows, cols, dev, dt)
    r, lddr = (None, 0) if dres is None else (dres.data_ptr(), _rows(dres, "dres", rows, cols, dev, dt))
    if dx is None:
        dx = _made((rows, cols), dt, dy.device, stream)
    lddx = _rows(dx, "dx", rows, cols, dev, dt)
    if want_params:
        dg = _made((cols,), torch.float32, dy.device, stream) if dg is None else dg
        db = _made((cols,), torch.float32, dy.device, stream) if db is None else db
    gp = None if dg is None else _vec(dg, "dg", cols, dev, _F32)
    bp = None if db is None else _vec(db, "db", cols, dev, _F32)
    w = (None, 0)
    if dg is not None or db is not None:
        w = _scratch(ws, gpt_layernorm_bwd_ws_bytes(rows, cols) if ws is None else 0, dev, dy.device, stream)
    st = lib().gpt_layernorm_bwd(dy.data_ptr(), lddy, h.data_ptr(), ldh, r, lddr, DT_BF16 if dt is _BF16 else DT_F32,
                                 _vec(g, "g", cols, dev, _FLOATS), _dt(g), _vec(mean, "mean", rows, dev, _F32),
                                 _vec(rstd, "rstd", rows, dev, _F32), rows, cols, dx.data_ptr(), lddx, gp, bp, *w,
                                 _stream_on(stream, dev))
    if st:
        _check("gpt_layernorm_bwd", st)
    return dx, dg, db


# ------------------------------------------------------------------ paged key/value cache
class CacheStruct(ctypes.Structure):
    """llama_cache of the C header."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("n_kv_heads", ctypes.c_int32),
                ("d_head", ctypes.c_int32), ("page_size", ctypes.c_int32), ("fmt", ctypes.c_int32)]


class SeqsStruct(ctypes.Structure):
    """llama_cache_seqs of the C header."""
    _fields_ = [("cu_rows", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("pages", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int64), ("max_pages", ctypes.c_int64), ("ld_pages", ctypes.c_int64)]


def _shaped(t: torch.Tensor, name: str, shape, dtype, device) -> torch.Tensor:
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor of shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, the rest on {device}")
    return t


CACHE_WS_COUNTS = 65536


class _Described:
    """An object whose C struct (address in _ref) holds the pointers and sizes of its
    attributes: those cannot be set to others, which the struct would not follow."""
    _fixed = frozenset()

    def __setattr__(self, name, value):
        if name in self._fixed and "_ref" in self.__dict__ and value is not self.__dict__.get(name):  # += sets the same one
            raise AttributeError(f"{type(self).__name__}.{name} cannot be replaced: copy into the tensor "
                                 f"(.copy_()), or make another {type(self).__name__}")
        object.__setattr__(self, name, value)

    def __delattr__(self, name):
        if name in self._fixed:
            raise AttributeError(f"{type(self).__name__}.{name} cannot be deleted")
        object.__delattr__(self, name)


class KVCache(_Described):
    """Pages of keys and values (llama_cache): fmt E4M3 or E5M2 (codes with one
    exponent byte per token and head, value = code * 2^(exp - 127)) or
    CACHE_BF16.  k [n_pages, n_kv_heads, page_size, d_head], v [n_pages,
    n_kv_heads, page_size / 16, d_head, 16], k_exp and v_exp [n_pages,
    n_kv_heads, page_size]; buffers that are not given are allocated, empty.  The
    tensors' contents may change, the attributes are those of the construction."""
    _fixed = frozenset(("k", "v", "k_exp", "v_exp", "n_pages", "n_kv_heads", "d_head", "page_size", "fmt", "device",
                        "_c", "_ref", "_dev"))

    def __init__(self, n_pages: int, n_kv_heads: int, d_head: int, page_size: int, fmt: int, device, k=None, v=None,
                 k_exp=None, v_exp=None):
        dev = torch.empty(0, device=device).device  # with its index
        self.device, self.fmt = dev, int(fmt)
        self.n_pages, self.n_kv_heads, self.d_head, self.page_size = n_pages, n_kv_heads, d_head, page_size
        dt = torch.bfloat16 if fmt == CACHE_BF16 else torch.uint8
        ks, vs = (n_pages, n_kv_heads, page_size, d_head), (n_pages, n_kv_heads, page_size // 16, d_head, 16)
        self.k = torch.empty(ks, dtype=dt, device=dev) if k is None else _shaped(k, "k", ks, dt, dev)
        self.v = torch.empty(vs, dtype=dt, device=dev) if v is None else _shaped(v, "v", vs, dt, dev)
        self.k_exp = self.v_exp = None
        if fmt != CACHE_BF16:
            es, u8 = ks[:3], torch.uint8
            self.k_exp = torch.empty(es, dtype=u8, device=dev) if k_exp is None else _shaped(k_exp, "k_exp", es, u8, dev)
            self.v_exp = torch.empty(es, dtype=u8, device=dev) if v_exp is None else _shaped(v_exp, "v_exp", es, u8, dev)
        self._c = CacheStruct(_p(self.k), _p(self.v), _p(self.k_exp), _p(self.v_exp), n_pages, n_kv_heads, d_head,
                              page_size, self.fmt)
        self._dev = self.k.get_device()
        self._ref = ctypes.addressof(self._c)


class CacheSeqs(_Described):
    """The sequences of a call (llama_cache_seqs), int32 device tensors: cu_rows
    [n + 1], kv_len [n] (tokens cached, the call's own included), pages [n,
    max_pages].  Their contents may change between calls (cu_rows.copy_(...)), the
    attributes are those of the construction."""
    _fixed = frozenset(("cu_rows", "kv_len", "pages", "n_seqs", "max_pages", "device", "_c", "_ref", "_dev"))

    def __init__(self, cu_rows: torch.Tensor, kv_len: torch.Tensor, pages: torch.Tensor):
        n = kv_len.numel()
        _shaped(kv_len, "kv_len", (n,), torch.int32, kv_len.device)
        _shaped(cu_rows, "cu_rows", (n + 1,), torch.int32, kv_len.device)
        if pages.dtype != torch.int32:
            raise TypeError(f"pages: expected torch.int32, got {pages.dtype}")
        if pages.dim() != 2 or pages.shape[0] != n or pages.device != kv_len.device:
            raise ValueError("pages: expected [n_seqs, max_pages] on the device of kv_len")
        self.cu_rows, self.kv_len, self.pages = cu_rows, kv_len, pages
        self.n_seqs, self.max_pages, self.device = n, pages.shape[1], kv_len.device
        self._c = SeqsStruct(_p(cu_rows), _p(kv_len), _p(pages), n, self.max_pages, _ld(pages))
        self._dev = kv_len.get_device()
        self._ref = ctypes.addressof(self._c)


def _cache_device(cache: KVCache, seqs: CacheSeqs) -> None:
    """The cache and the sequences are on the current GPU (its stream runs the call)."""
    dev = cache._dev
    if dev < 0 or seqs._dev != dev or _current() != dev:
        raise ValueError(f"the cache is on {cache.device}, the sequences on {seqs.device}: "
                         "both must be on the current GPU")


def _mat(t: torch.Tensor, name: str, rows: int, cols: int, dev: int) -> int:
    """Row stride of a bf16 tensor [rows or more, cols] with contiguous rows on GPU
    dev.  (A call of these is a few microseconds of host work: one look at each
    property.)"""
    if t.dtype is not _BF16:
        raise TypeError(f"{name}: expected bfloat16, got {t.dtype}")
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or shape[0] < rows or shape[1] != cols or (stride[1] != 1 and cols > 1):
        raise ValueError(f"{name}: expected [{rows}, {cols}] with contiguous rows, got {tuple(shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name}: on {t.device}, the cache on GPU {dev}")
    return stride[0] if shape[0] > 1 else max(cols, 1)


def _new(rows: int, cols: int, device, stream) -> torch.Tensor:
    """bf16 output [rows, cols] of a call, of the memory of the stream that writes it."""
    if stream is None:
        return torch.empty((rows, cols), dtype=_BF16, device=device)
    with torch.cuda.stream(stream):
        return torch.empty((rows, cols), dtype=_BF16, device=device)


def llama_cache_append(qkv, cache: KVCache, seqs: CacheSeqs, n_heads: int, table=None, q=None, stream=None):
    """Rotate the queries and keys of the call's rows (table: llama_rope_table of
    at least max_pages * page_size positions; None: no rotation) and write keys
    and values into the cache.  qkv: [rows, (n_heads + 2 n_kv_heads) d_head].
    q: [rows, n_heads d_head], may be a view of qkv's query columns.  Returns q."""
    dev = cache._dev
    rows, dh = qkv.shape[0], cache.d_head
    ld = _mat(qkv, "qkv", rows, (n_heads + 2 * cache.n_kv_heads) * dh, dev)
    if q is None:
        q = _new(rows, n_heads * dh, qkv.device, stream)
    ldq = _mat(q, "q", rows, n_heads * dh, dev)
    tp, tn = None, 0
    if table is not None:
        if table.dtype is not torch.float32 or not table.is_contiguous():
            raise TypeError("table: expected a contiguous float32 tensor")
        if table.get_device() != dev:
            raise ValueError(f"table: on {table.device}, the cache on GPU {dev}")
        tp, tn = table.data_ptr(), table.numel() // dh
    _cache_device(cache, seqs)
    st = lib().llama_cache_append(qkv.data_ptr(), rows, ld, n_heads, cache._ref, seqs._ref, tp, tn, q.data_ptr(), ldq,
                                  _stream(stream))
    if st:
        _check("llama_cache_append", st)
    return q


def llama_cache_read(cache: KVCache, seqs: CacheSeqs, rows: int, k=None, v=None, want_k=True, want_v=True,
                     stream=None):
    """Cached keys and values of the positions that the call's rows stand for, as
    bf16 [rows, n_kv_heads d_head].  Returns (k, v)."""
    dev = cache._dev
    cols = cache.n_kv_heads * cache.d_head
    if want_k and k is None:
        k = _new(rows, cols, cache.device, stream)
    if want_v and v is None:
        v = _new(rows, cols, cache.device, stream)
    ldk = _mat(k, "k", rows, cols, dev) if k is not None else 0
    ldv = _mat(v, "v", rows, cols, dev) if v is not None else 0
    _cache_device(cache, seqs)
    st = lib().llama_cache_read(cache._ref, seqs._ref, rows, _p(k), ldk, _p(v), ldv, _stream(stream))
    if st:
        _check("llama_cache_read", st)
    return k, v


def llama_cache_attention_ws_bytes(rows: int, n_heads: int, cache: KVCache, seqs: CacheSeqs, max_rows: int) -> int:
    return int(lib().llama_cache_attention_ws_bytes(int(rows), int(n_heads), cache._ref, seqs._ref, int(max_rows)))


def cache_attention_workspace(rows: int, n_heads: int, cache: KVCache, seqs: CacheSeqs, max_rows: int) -> torch.Tensor:
    """Workspace of llama_cache_attention: its counters are zero, and left zero by
    every completed call of it; other calls must not write it, unless it is only
    used with a fused quantise (one per stream of concurrent calls).  The zeros are
    written on the current stream: a first call on another one has to wait for it."""
    ws = torch.empty(max(llama_cache_attention_ws_bytes(rows, n_heads, cache, seqs, max_rows), CACHE_WS_COUNTS),
                     dtype=torch.uint8, device=cache.device)
    ws[:CACHE_WS_COUNTS].zero_()
    return ws


def llama_cache_attention(q, cache: KVCache, seqs: CacheSeqs, n_heads: int, max_rows: int, window: int = 0, o=None,
                          fq: FusedQuant | None = None, ws=None, stream=None):
    """Causal grouped-query attention of the call's rows (q [rows, n_heads
    d_head]) over the cache, optionally with the fused quantise of o (its ws, of
    llama_cache_attention_ws_bytes and shared with other fused calls if wanted, is
    then the call's; without either one is made for the call, on the current stream
    only).  max_rows: at least the rows of every sequence.  Returns o."""
    dev = cache._dev
    rows, cols = q.shape[0], n_heads * cache.d_head
    ldq = _mat(q, "q", rows, cols, dev)
    if o is None:
        o = _new(rows, cols, q.device, stream)
    ldo = _mat(o, "o", rows, cols, dev)
    quant = _NO_QUANT[:-2]
    _cache_device(cache, seqs)
    if fq is not None:
        ws, quant = fq.ws, fq.args()[:-2]
        if fq.q.shape != (rows, cols) or fq.q.dtype != torch.uint8 or fq.q.stride(1) != 1:
            raise ValueError(f"fq.q: expected uint8 [{rows}, {cols}] with contiguous rows")
        if any(t is not None and t.get_device() != dev for t in (fq.q, fq.bias, fq.bias_pred, fq.amax_bits, fq.flags)):
            raise ValueError(f"fq: every tensor must be on GPU {dev}")
    elif ws is None:
        if stream is not None:  # its zeros are written on the current stream, and its memory is that one's
            raise ValueError("ws: a call on a stream of the caller's needs a workspace")
        ws = cache_attention_workspace(rows, n_heads, cache, seqs, max_rows)
    if ws.get_device() != dev:
        raise ValueError(f"ws: on {ws.device}, the cache on GPU {dev}")
    if not ws.is_contiguous():  # an expanded one is shorter than its elements
        raise ValueError("ws: expected a contiguous tensor")
    st = lib().llama_cache_attention(q.data_ptr(), rows, ldq, n_heads, cache._ref, seqs._ref, max_rows, window,
                                     o.data_ptr(), ldo, *quant, ws.data_ptr(), ws.numel() * ws.element_size(),
                                     _stream(stream))
    if st:
        _check("llama_cache_attention", st)
    return o
