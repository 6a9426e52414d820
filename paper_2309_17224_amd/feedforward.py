"""The feed-forward blocks around the FP8 linears, as library calls.

The models the paper trains and runs have two kinds (Table 1): the GPT block,
with a layer norm, biases, GELU and a residual sum, and Llama 2's gated block.
Their linears are FP8 with one FP8-AMAX bias per tensor (Sec. 2.3 Eq. 3, Sec. 3):
weights and activations E4M3, gradients E5M2 (Sec. 2.2); the rest is in bf16 with
fp32 arithmetic, in the epilogues of the matmuls where it follows one:

  GPT      xn = LayerNorm(h) g + b                      -> codes
           z = xn8 . W1_8 + b1;  a = act(z)             -> codes      (one matmul call)
           out = h + a8 . W2_8 + b2                                   (one matmul call)
  gated    (g | u) = x8 . Wgu_8;  a = act(g) u          -> codes      (one matmul call)
           y = a8 . Wd_8

and backward
  GPT      db2 = sum dout;  dz = (dout8 . W2_8^T) act'(z) -> codes, db1 = sum dz  (one matmul call)
           dW2 = a8^T . dout8;  dxn = dz8 . W1_8^T;  dW1 = xn8^T . dz8
           dh = LayerNorm'(dxn) + dout, dg, db
  gated    t = dy8 . Wd_8^T;  dg = t u act'(g), du = t act(g) -> codes            (one matmul call)
           dWd = a8^T . dy8;  dx = dgu8 . Wgu_8^T;  dWgu = x8^T . dgu8

Each fused quantise casts with the previous call's bias as a prediction and casts
again only if the exact bias differs, so the codes are always those of the exact
bias.  Every buffer is allocated once; a call launches kernels only and can be
captured in a HIP graph.
"""
from __future__ import annotations

import gc

import torch

from . import fp8lin as F
from .linear import Fp8Tensor

BF16 = torch.bfloat16


def _index(dev: torch.device) -> int:
    """The GPU of a device, -1 of the host."""
    return dev.index if dev.type == "cuda" else -1


class _Block:
    """Buffers shared by the two blocks: FP8 forms of tensors, each with its workspace."""

    def __init__(self, rows: int, device, act: int, train: bool):
        if rows < 1:
            raise ValueError(f"rows: at least one token, got {rows}")
        if act not in (F.ACT_NONE, F.ACT_RELU, F.ACT_GELU, F.ACT_GELU_TANH, F.ACT_SILU):
            raise ValueError(f"act: expected one of the ACT_ constants, got {act}")
        self.rows, self.act, self.train = rows, act, train
        self.dev = torch.empty(0, device=device).device
        self.graph = None
        self.weighed = self.ran = False  # set_weights, and then forward, have run

    def _new(self, *shape, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=self.dev)

    def _fp8(self, rows: int, cols: int, transposed: bool = True, plain: bool = True) -> Fp8Tensor:
        t = Fp8Tensor(rows, cols, self.dev, want_q=plain, want_qT=transposed)
        t.qws = self._new(max(F.fp8_linear_quantise_ws_bytes(rows, cols), F.fp8_quantise_ws_bytes(rows, cols),
                              F.gpt_layernorm_ws_bytes(rows), 4), dtype=torch.uint8)
        return t

    @staticmethod
    def _fq(t: Fp8Tensor, fmt: int) -> F.FusedQuant:
        return F.FusedQuant(t.q, t.bias, t.qws, fmt, bias_pred=t.bias, amax_bits=t.amax, flags=t.flags, qT=t.qT)

    @staticmethod
    def _quantise(x: torch.Tensor, t: Fp8Tensor, fmt: int, predict: bool = True) -> None:
        F.fp8_quantise(x, fmt, 0, bias_pred=t.bias if predict else None, bias=t.bias, amax_bits=t.amax, flags=t.flags,
                       q=t.q, qT=t.qT, want_q=t.q is not None, want_qT=t.qT is not None, ws=t.qws)

    def _on_current_gpu(self) -> None:
        """The calls of a block run on the current GPU's stream."""
        gpu = _index(self.dev)
        if gpu >= 0 and F._current() != gpu:
            raise ValueError(f"the block is on {self.dev}, which is not the current GPU")

    def _take(self, x: torch.Tensor, name: str, cols: int) -> torch.Tensor:
        self._on_current_gpu()
        if x.shape != (self.rows, cols) or x.dtype != BF16 or x.device != self.dev:
            raise ValueError(f"{name}: expected bfloat16 [{self.rows}, {cols}] on {self.dev}, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
        return x

    def _check(self, x: torch.Tensor, name: str, *shape: int) -> None:
        """A weight (its rows contiguous), bias or gain that a call can take."""
        self._on_current_gpu()
        if tuple(x.shape) != shape or x.device != self.dev:
            raise ValueError(f"{name}: expected {shape} on {self.dev}, got {tuple(x.shape)} on {x.device}")
        if x.dtype not in (BF16, torch.float32):
            raise TypeError(f"{name}: expected bfloat16 or float32, got {x.dtype}")
        rows, cols = shape if len(shape) == 2 else (1, 1)
        if (cols > 1 and x.stride(1) != 1) or (rows > 1 and x.stride(0) < cols):
            raise ValueError(f"{name}: expected contiguous rows that do not overlap, got strides {x.stride()}")

    def _own(self, name: str, x: torch.Tensor) -> None:
        """x copied into the block's tensor of that name, whose address a captured graph has."""
        t = getattr(self, name, None)
        if t is None:
            setattr(self, name, x.detach().clone(memory_format=torch.contiguous_format))
        else:
            t.copy_(x.detach())  # of a parameter the values alone, without an autograd history

    def _needs_weights(self) -> None:
        if not self.weighed:
            raise RuntimeError("forward: the block has no weights yet (set_weights)")

    def _needs_training(self) -> None:
        if not self.train:
            raise RuntimeError("this block was made for inference (train=False)")
        if not self.ran:
            raise RuntimeError("backward: no forward has run yet")

    def capture(self, step):
        """Record step() (calls of this block, on tensors that stay) into a HIP graph;
        replay() launches it again on those tensors' current contents.  step() has to
        have run once before."""
        torch.cuda.synchronize(self.dev)
        g = torch.cuda.CUDAGraph()
        gc.collect()  # dead objects that own graphs must not be destroyed during the capture
        was_enabled = gc.isenabled()
        gc.disable()
        try:
            with torch.cuda.graph(g):
                step()
        finally:
            if was_enabled:
                gc.enable()
        torch.cuda.synchronize(self.dev)
        self.graph = g
        return g

    def replay(self) -> None:
        if self.graph is None:
            raise RuntimeError("replay: nothing was recorded yet (capture)")
        self.graph.replay()


class GptFeedForward(_Block):
    """out = h + act(LayerNorm(h) W1 + b1) W2 + b2 for `rows` tokens of d columns.

    set_weights(W1 [d, ffn], b1 [ffn], W2 [ffn, d], b2 [d], g [d], b [d]) casts the
    weights and copies the rest, after every update (a captured graph follows it); each
    bf16 or fp32, g and b of one type, biases and gain of the types of the first time.
    forward(h) returns out; h has to stay as it is until backward.  backward(dout)
    returns dh and leaves dw1, dw2, dg, db (fp32) and db1, db2 (of the biases' type)."""

    def __init__(self, rows: int, d: int, ffn: int, device, act: int = F.ACT_GELU, eps: float = 1e-5, train: bool = True):
        super().__init__(rows, device, act, train)
        self.d, self.ffn, self.eps = d, ffn, float(eps)
        self.w1, self.w2 = self._fp8(d, ffn, plain=train), self._fp8(ffn, d, plain=train)
        self.xn, self.a, self.out = self._new(rows, d), self._new(rows, ffn), self._new(rows, d)
        self.xn8, self.a8 = self._fp8(rows, d, transposed=train), self._fp8(rows, ffn, transposed=train)
        self.z = self.mean = self.rstd = self.db1 = self.db2 = None
        if train:
            f32 = torch.float32
            self.z, self.mean, self.rstd = self._new(rows, ffn), self._new(rows, dtype=f32), self._new(rows, dtype=f32)
            self.dout8, self.dz8 = self._fp8(rows, d), self._fp8(rows, ffn)
            self.dz, self.dxn, self.dh = self._new(rows, ffn), self._new(rows, d), self._new(rows, d)
            self.dw1, self.dw2 = self._new(d, ffn, dtype=f32), self._new(ffn, d, dtype=f32)
            self.dg, self.db = self._new(d, dtype=f32), self._new(d, dtype=f32)
            self.sums = torch.empty(max(F.gpt_bias_grad_ws_bytes(rows, ffn), F.gpt_bias_grad_ws_bytes(rows, d),
                                        F.gpt_layernorm_bwd_ws_bytes(rows, d)), dtype=torch.uint8, device=self.dev)

    def set_weights(self, W1, b1, W2, b2, g, b) -> None:
        d, ffn = self.d, self.ffn
        for x, name, shape in ((W1, "W1", (d, ffn)), (b1, "b1", (ffn,)), (W2, "W2", (ffn, d)), (b2, "b2", (d,)),
                               (g, "g", (d,)), (b, "b", (d,))):
            self._check(x, name, *shape)
        if g.dtype != b.dtype:
            raise TypeError(f"g and b: expected one type, got {g.dtype} and {b.dtype}")
        for name, x in (("b1", b1), ("b2", b2), ("g", g), ("b", b)):
            t = getattr(self, name, None)
            if t is not None and t.dtype != x.dtype:
                raise TypeError(f"{name}: the block was set up with {t.dtype}, got {x.dtype}")
        for name, x in (("b1", b1), ("b2", b2), ("g", g), ("b", b)):
            self._own(name, x)
        if self.train and self.db1 is None:
            self.db1, self.db2 = torch.empty_like(self.b1), torch.empty_like(self.b2)
        self._quantise(W1, self.w1, F.E4M3, predict=False)
        self._quantise(W2, self.w2, F.E4M3, predict=False)
        self.weighed = True

    def forward(self, h: torch.Tensor) -> torch.Tensor:
        self._needs_weights()
        self._take(h, "h", self.d)
        if self.train and h.untyped_storage().data_ptr() == self.out.untyped_storage().data_ptr():
            raise ValueError("h: the block's own output, which this call overwrites before backward reads it")
        # the layer norm casts its rows itself where no transposed codes are needed
        F.gpt_layernorm_quantise(h, self.g, self.b, self.eps, y=self.xn, mean=self.mean, rstd=self.rstd,
                                 fq=None if self.train else self._fq(self.xn8, F.E4M3))
        if self.train:
            self._quantise(self.xn, self.xn8, F.E4M3)
        F.fp8_linear_fwd_act(self.xn8.q, self.xn8.bias, self.w1.qT, self.w1.bias, self.act, bias=self.b1, z=self.z, y=self.a,
                             fq=self._fq(self.a8, F.E4M3))
        F.fp8_linear_fwd_act(self.a8.q, self.a8.bias, self.w2.qT, self.w2.bias, F.ACT_NONE, bias=self.b2, res=h, y=self.out)
        self.h, self.ran = h, True
        return self.out

    def backward(self, dout: torch.Tensor) -> torch.Tensor:
        self._needs_training()
        self._take(dout, "dout", self.d)
        self._quantise(dout, self.dout8, F.E5M2)
        F.gpt_bias_grad(dout, db=self.db2, ws=self.sums)
        F.fp8_linear_bwd_dx_act(self.dout8.q, self.dout8.bias, self.w2.q, self.w2.bias, self.z, self.act, dz=self.dz,
                                db=self.db1, fq=self._fq(self.dz8, F.E5M2), ws=self.sums)
        F.fp8_linear_bwd_dw(self.a8.qT, self.a8.bias, self.dout8.qT, self.dout8.bias, dw=self.dw2)
        F.fp8_linear_bwd_dx(self.dz8.q, self.dz8.bias, self.w1.q, self.w1.bias, dx=self.dxn)
        F.fp8_linear_bwd_dw(self.xn8.qT, self.xn8.bias, self.dz8.qT, self.dz8.bias, dw=self.dw1)
        F.gpt_layernorm_bwd(self.dxn, self.h, self.g, self.mean, self.rstd, dres=dout, dx=self.dh, dg=self.dg, db=self.db,
                            ws=self.sums)
        return self.dh


class GatedFeedForward(_Block):
    """y = (act(x Wg) * (x Wu)) Wd for `rows` tokens of d columns.

    set_weights(Wgu [d, 2 ffn] (gate columns first), Wd [ffn, d]) casts the weights.
    forward(x) returns y; backward(dy) returns dx and leaves dwgu and dwd (fp32)."""

    def __init__(self, rows: int, d: int, ffn: int, device, act: int = F.ACT_SILU, train: bool = True):
        super().__init__(rows, device, act, train)
        self.d, self.ffn = d, ffn
        self.wgu, self.wd = self._fp8(d, 2 * ffn, plain=train), self._fp8(ffn, d, plain=train)
        self.a, self.y = self._new(rows, ffn), self._new(rows, d)
        self.x8, self.a8 = self._fp8(rows, d, transposed=train), self._fp8(rows, ffn, transposed=train)
        self.gu = None
        if train:
            self.gu, self.dgu, self.dx = self._new(rows, 2 * ffn), self._new(rows, 2 * ffn), self._new(rows, d)
            self.dy8, self.dgu8 = self._fp8(rows, d), self._fp8(rows, 2 * ffn)
            self.dwgu, self.dwd = self._new(d, 2 * ffn, dtype=torch.float32), self._new(ffn, d, dtype=torch.float32)

    def set_weights(self, Wgu, Wd) -> None:
        self._check(Wgu, "Wgu", self.d, 2 * self.ffn)
        self._check(Wd, "Wd", self.ffn, self.d)
        self._quantise(Wgu, self.wgu, F.E4M3, predict=False)
        self._quantise(Wd, self.wd, F.E4M3, predict=False)
        self.weighed = True

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        self._needs_weights()
        self._quantise(self._take(x, "x", self.d), self.x8, F.E4M3)
        F.fp8_linear_fwd_glu(self.x8.q, self.x8.bias, self.wgu.qT, self.wgu.bias, self.act, gu=self.gu, a=self.a,
                             fq=self._fq(self.a8, F.E4M3))
        F.fp8_linear_fwd(self.a8.q, self.a8.bias, self.wd.qT, self.wd.bias, y=self.y)
        self.ran = True
        return self.y

    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        self._needs_training()
        self._quantise(self._take(dy, "dy", self.d), self.dy8, F.E5M2)
        F.fp8_linear_bwd_dx_glu(self.dy8.q, self.dy8.bias, self.wd.q, self.wd.bias, self.gu, self.act, dgu=self.dgu,
                                fq=self._fq(self.dgu8, F.E5M2))
        F.fp8_linear_bwd_dw(self.a8.qT, self.a8.bias, self.dy8.qT, self.dy8.bias, dw=self.dwd)
        F.fp8_linear_bwd_dx(self.dgu8.q, self.dgu8.bias, self.wgu.q, self.wgu.bias, dx=self.dx)
        F.fp8_linear_bwd_dw(self.x8.qT, self.x8.bias, self.dgu8.qT, self.dgu8.bias, dw=self.dwgu)
        return self.dx
