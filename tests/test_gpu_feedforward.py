"""The feed-forward blocks (GptFeedForward, GatedFeedForward) and the decoder layer
over the gated matmul: the operators run together, forward, backward and captured.

Stage by stage against the oracle in fp64, each stage on the codes that the block
itself made for it (so that a code that another rounding moves is no difference):
biases and codes are those of fp8_quantise of the stage's bf16 input, bit for bit,
and each output is within its bound: for a matmul 2^-11 of the sum of the products'
magnitudes (the matrix core) and half a step of the output, with the epilogue's own
bounds (test_gpu_ffn.py); for the layer norm its arithmetic (test_gpu_layernorm.py).
"""
import numpy as np
import pytest
import torch

from oracle import ffn as O
from paper_2309_17224_amd import decoder as DL
from paper_2309_17224_amd import feedforward as FF
from paper_2309_17224_amd import fp8lin as F
from paper_2309_17224_amd import workloads as wl
from parity_util import np_bits, rel_f
from test_gpu_ffn import ACT, E4, E5, close, sums_bound
from test_gpu_layernorm import S, U, stat_errors

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def f64(t):
    return t.double().cpu().numpy()


def value(t, kind, transposed=False):
    """What an Fp8Tensor's codes stand for."""
    q = t.qT.t() if transposed else t.q
    return q.view(kind).double().cpu().numpy() * 2.0 ** -int(t.bias)


def same_codes(t, x, kind):
    fmt = F.E4M3 if kind is E4 else F.E5M2
    q, qT, bias, amax, flags = F.fp8_quantise(x, fmt, want_qT=True)
    assert int(t.bias) == int(bias) and int(t.amax) == int(amax) and int(t.flags) == int(flags)
    if t.q is not None:
        assert torch.equal(t.q, q)
    if t.qT is not None:
        assert torch.equal(t.qT, qT)


def product(a, b):
    """A [M, K] . B [K, N] in fp64 and the matrix core's bound."""
    return a @ b, sums_bound(a, b.T, 1.0)


def gpt(gpu, rows, d, ffn, act, seed, train=True, std=0.05):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    block = FF.GptFeedForward(rows, d, ffn, gpu, act=act, train=train)
    w = dict(W1=(std * r(d, ffn)).to(BF), b1=(0.2 * r(ffn)).to(BF), W2=(std * r(ffn, d)).to(BF), b2=(0.2 * r(d)).to(BF),
             g=(1 + 0.1 * r(d)).to(BF), b=(0.1 * r(d)).to(BF))
    block.set_weights(**{k: v.to(gpu) for k, v in w.items()})
    return block, w, (r(rows, d) + 0.2).to(BF).to(gpu), (1e-3 * r(rows, d)).to(BF).to(gpu)


def check_norm(block, h, w):
    y, m, s = O.layernorm(f64(h), f64(w["g"]), f64(w["b"]), 1e-5)
    dm, ds = stat_errors(f64(h), m, s)
    xh, gv = np.abs(f64(h) - m[:, None]) * s[:, None], np.abs(f64(w["g"]))
    close(block.xn, y, gv * (xh * (ds[:, None] + 4 * U) + dm[:, None] * s[:, None]) + 2 * U * (np.abs(y) + gv * xh), BF)


def check_act(out, z, ez, act, extra=0.0, dt=BF):
    f = O.act(z, act)
    close(out, f + extra, O.SLOPE_MAX[act] * ez + 2.0 ** -18 * np.abs(f) + 1e-9 + 2.0 ** -24 * np.abs(f + extra), dt)


@pytest.mark.parametrize("rows,d,ffn,act", [(1, 96, 200, "gelu"), (33, 512, 1408, "gelu_tanh"), (300, 136, 520, "relu"),
                                            (700, 2048, 4096, "gelu")], ids=str)
def test_gpt_block(gpu, rows, d, ffn, act):
    block, w, h, dout = gpt(gpu, rows, d, ffn, ACT[act], rows)
    for turn in range(2):                     # the second with predictions that hold
        out = block.forward(h)
        dh = block.backward(dout)
    check_norm(block, h, w)
    same_codes(block.xn8, block.xn, E4)
    same_codes(block.w1, w["W1"].to(gpu), E4)
    W1, W2 = value(block.w1, E4), value(block.w2, E4)
    z, ez = product(value(block.xn8, E4), W1)
    z = z + f64(w["b1"])
    close(block.z, z, ez + 2.0 ** -23 * np.abs(z), BF)
    check_act(block.a, z, ez + 2.0 ** -23 * np.abs(z), act)
    same_codes(block.a8, block.a, E4)
    y, ey = product(value(block.a8, E4), W2)
    y = y + f64(w["b2"]) + f64(h)
    close(out, y, ey + 2.0 ** -22 * (np.abs(y) + np.abs(f64(h))), BF)
    # backward
    same_codes(block.dout8, dout, E5)
    g8 = value(block.dout8, E5)
    mags = np.abs(f64(dout)).sum(axis=0)
    close(block.db2, f64(dout).sum(axis=0), (rows + 24) * U * mags, BF)
    t, et = product(g8, W2.T)
    sl = O.slope(f64(block.z), act)
    err = et * np.abs(sl) + 2.0 ** -18 * np.abs(t)
    close(block.dz, t * sl, err, BF)
    close(block.db1, (t * sl).sum(axis=0), err.sum(axis=0) + rows * U * (np.abs(t * sl) + err).sum(axis=0), BF)
    same_codes(block.dz8, block.dz, E5)
    for got, a, b in ((block.dw2, value(block.a8, E4, True).T, g8),
                      (block.dw1, value(block.xn8, E4, True).T, value(block.dz8, E5, True))):
        ref, e = product(a, b)
        close(got, ref, e + U * np.abs(ref), F32)
    dxn, e = product(value(block.dz8, E5), W1.T)
    close(block.dxn, dxn, e, BF)
    hv, gv, m, s = f64(h), f64(w["g"]), f64(block.mean), f64(block.rstd)
    rdx, rdg, rdb = O.layernorm_bwd(f64(block.dxn), hv, gv, m, s, f64(dout))
    xh, wv = (hv - m[:, None]) * s[:, None], f64(block.dxn) * gv
    c1, c2 = np.abs(wv).mean(axis=1)[:, None], np.abs(wv * xh).mean(axis=1)[:, None]
    n = S(d) + 12 * U
    close(dh, rdx, s[:, None] * n * (np.abs(wv) + c1 + np.abs(xh) * c2) + U * (np.abs(rdx) + np.abs(f64(dout))), BF)
    close(block.dg, rdg, (rows + 27) * U * np.abs(f64(block.dxn) * xh).sum(axis=0), F32)
    close(block.db, rdb, (rows + 24) * U * np.abs(f64(block.dxn)).sum(axis=0), F32)


@pytest.mark.parametrize("rows,d,ffn,act", [(1, 96, 200, "silu"), (33, 512, 1408, "silu"), (300, 136, 520, "gelu"),
                                            (700, 2048, 4096, "silu")], ids=str)
def test_gated_block(gpu, rows, d, ffn, act):
    g = torch.Generator().manual_seed(rows)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    block = FF.GatedFeedForward(rows, d, ffn, gpu, act=ACT[act])
    Wgu, Wd = (0.05 * r(d, 2 * ffn)).to(BF).to(gpu), (0.05 * r(ffn, d)).to(BF).to(gpu)
    block.set_weights(Wgu, Wd)
    x, dy = r(rows, d).to(BF).to(gpu), (1e-3 * r(rows, d)).to(BF).to(gpu)
    for turn in range(2):
        y = block.forward(x)
        dx = block.backward(dy)
    same_codes(block.x8, x, E4)
    same_codes(block.wgu, Wgu, E4)
    W, D = value(block.wgu, E4), value(block.wd, E4)
    z, ez = product(value(block.x8, E4), W)
    ez = ez + 2.0 ** -23 * np.abs(z)
    close(block.gu, z, ez, BF)
    gate, up = z[:, :ffn], z[:, ffn:]
    f = O.act(gate, act)
    eg, eu = O.SLOPE_MAX[act] * ez[:, :ffn] + 2.0 ** -18 * np.abs(f) + 1e-9, ez[:, ffn:]
    close(block.a, f * up, eg * np.abs(up) + eu * np.abs(f) + eg * eu + U * np.abs(f * up), BF)
    same_codes(block.a8, block.a, E4)
    ref, e = product(value(block.a8, E4), D)
    close(y, ref, e, BF)
    same_codes(block.dy8, dy, E5)
    t, et = product(value(block.dy8, E5), D.T)
    gub = f64(block.gu)
    gate, up = gub[:, :ffn], gub[:, ffn:]
    sl, f = O.slope(gate, act), O.act(gate, act)
    err = np.concatenate([et * np.abs(sl * up) + 2.0 ** -18 * np.abs(t * up), et * np.abs(f) + np.abs(t) * (2.0 ** -18 * np.abs(f) + 1e-9)], axis=1)
    close(block.dgu, np.concatenate([t * up * sl, t * f], axis=1), err, BF)
    same_codes(block.dgu8, block.dgu, E5)
    for got, a, b in ((block.dwd, value(block.a8, E4, True).T, value(block.dy8, E5, True)),
                      (block.dwgu, value(block.x8, E4, True).T, value(block.dgu8, E5, True))):
        ref, e = product(a, b)
        close(got, ref, e + U * np.abs(ref), F32)
    ref, e = product(value(block.dgu8, E5), W.T)
    close(dx, ref, e, BF)


@pytest.mark.parametrize("rows", [1, 5, 300])
def test_inference_blocks_give_the_training_blocks_bits(gpu, rows):
    """Without what only the backward pass needs, the outputs are the same."""
    block, w, h, _ = gpt(gpu, rows, 256, 768, F.ACT_GELU, 3)
    infer = gpt(gpu, rows, 256, 768, F.ACT_GELU, 3, train=False)[0]
    assert torch.equal(infer.forward(h), block.forward(h))
    assert torch.equal(infer.a8.q, block.a8.q) and torch.equal(infer.xn8.q, block.xn8.q)
    a, b = (FF.GatedFeedForward(rows, 256, 768, gpu, train=t) for t in (True, False))
    g = torch.Generator().manual_seed(4)
    Wgu, Wd = ((0.05 * torch.randn(*s, generator=g)).to(BF).to(gpu) for s in ((256, 1536), (768, 256)))
    for m in (a, b):
        m.set_weights(Wgu, Wd)
    assert torch.equal(a.forward(h), b.forward(h)) and torch.equal(a.a8.q, b.a8.q)
    with pytest.raises(RuntimeError):
        infer.backward(h)
    with pytest.raises(RuntimeError):
        b.backward(h)


@pytest.mark.parametrize("rows", [40, 600])
@pytest.mark.parametrize("kind", ["gpt", "gated"])
def test_captured_step_follows_its_inputs(gpu, rows, kind):
    """A captured step, replayed with other inputs between the program's own eager work
    on another block, gives the eager bits every time; two graphs live side by side."""
    d, ffn = 512, 2048

    def make():
        if kind == "gpt":
            return gpt(gpu, rows, d, ffn, F.ACT_GELU, 7)[0]
        g = torch.Generator().manual_seed(7)
        m = FF.GatedFeedForward(rows, d, ffn, gpu)
        m.set_weights(*((0.05 * torch.randn(*s, generator=g)).to(BF).to(gpu) for s in ((d, 2 * ffn), (ffn, d))))
        return m

    eager, first, second = make(), make(), make()
    xs = [torch.zeros((rows, d), dtype=BF, device=gpu) for _ in range(2)]
    dys = [torch.zeros((rows, d), dtype=BF, device=gpu) for _ in range(2)]
    g = torch.Generator().manual_seed(8)
    data = [((torch.randn(rows, d, generator=g) * (1 + i)).to(BF).to(gpu), (10.0 ** -i * torch.randn(rows, d, generator=g)).to(BF).to(gpu))
            for i in range(4)]

    def step(m, x, dy):
        def run():
            m.forward(x)
            m.backward(dy)
        return run

    for m, x, dy in ((first, xs[0], dys[0]), (second, xs[1], dys[1])):
        x.copy_(data[0][0])
        dy.copy_(data[0][1])
        step(m, x, dy)()
        m.capture(step(m, x, dy))
    outs = ("out", "dh", "dw1", "dw2", "db1", "db2", "dg", "db") if kind == "gpt" else ("y", "dx", "dwgu", "dwd")
    for turn in range(4):
        for k, m in enumerate((first, second)):
            x, dy = data[(turn + k) % 4]
            xs[k].copy_(x)
            dys[k].copy_(dy)
            m.replay()
        for k, m in enumerate((first, second)):
            step(eager, *data[(turn + k) % 4])()
            for name in outs:
                assert torch.equal(getattr(m, name), getattr(eager, name)), (turn, k, name)
        torch.cuda.synchronize()


def test_blocks_refuse(gpu):
    block, w, h, dout = gpt(gpu, 4, 64, 128, F.ACT_GELU, 1)
    for bad in (h[:3], h.float(), h.cpu(), torch.zeros((4, 65), dtype=BF, device=gpu)):
        with pytest.raises((ValueError, TypeError)):
            block.forward(bad)
    with pytest.raises(ValueError):
        block.set_weights(**{**{k: v.to(gpu) for k, v in w.items()}, "b1": w["b2"].to(gpu)})
    with pytest.raises(ValueError):
        FF.GptFeedForward(0, 64, 128, gpu)
    with pytest.raises(ValueError):
        FF.GatedFeedForward(4, 64, 128, gpu, act=9)
    with pytest.raises(ValueError):
        DL.DecoderLayer(wl.LAYERS["tiny-layer"], {}, gpu, bias_per="sequence", fused_glu=True)


# ------------------------------------------------------------------ the decoder layer over the gated matmul
def layers(gpu, **kw):
    cfg = wl.LAYERS["tiny-layer"]
    T = {t.name: wl.make_layer_tensor(cfg, t.name) for t in cfg.tensors()}
    W = {k: v.to(gpu) for k, v in T.items() if k != "H"}
    return cfg, T, [DL.DecoderLayer(cfg, W, gpu, **k) for k in ({}, kw)]


def test_decoder_layer_over_the_gated_matmul(gpu):
    """Same codes in, the gated matmul's a within a bf16 rounding of gate and up (2^-8 of
    each, which the activation's slope, at most 1.1 times |up|, and its value pass on) and of
    the unfused call's; the layer's output within the bar of an FP8 chain (2^-4)."""
    cfg, T, (plain, fused) = layers(gpu, fused_glu=True)
    for m in (plain, fused):
        m.H.copy_(T["H"].to(gpu))
        m.run()
        m.run()
    assert fused.gu is None and torch.equal(fused.hn.q, plain.hn.q)
    gate, up = f64(plain.gu)[:, :cfg.ffn], f64(plain.gu)[:, cfg.ffn:]
    bound = 2.0 ** -8 * (1.1 * np.abs(gate * up) + np.abs(O.act(gate, "silu") * up)) * 1.02
    close(fused.act.x, f64(plain.act.x), bound + 2.0 ** -8 * np.abs(f64(plain.act.x)), BF)
    q, _, bias, amax, _ = F.fp8_quantise(fused.act.x, F.E4M3)
    assert torch.equal(fused.act.q, q) and int(fused.act.bias) == int(bias)
    assert rel_f(np_bits(fused.out), np_bits(plain.out)) <= 2.0 ** -4
    want = fused.out.clone()
    fused.capture()
    for _ in range(3):
        fused.out.zero_()
        fused.replay()
        assert torch.equal(fused.out, want)
        plain.run()


def test_cached_layer_over_the_gated_matmul(gpu):
    """Prefill and single tokens through the cache: the layer's own bits against the
    layer without a cache, up to the attention's roundings."""
    cfg = wl.LAYERS["tiny-layer"]
    T = {t.name: wl.make_layer_tensor(cfg, t.name) for t in cfg.tensors()}
    W = {k: v.to(gpu) for k, v in T.items() if k != "H"}
    outs = []
    for fused in (False, True):
        m = DL.CachedDecoderLayer(cfg, W, gpu, n_seqs=2, max_pages=4, page_size=64, kv_fmt=F.CACHE_BF16, fused_glu=fused)
        m.H.copy_(T["H"].to(gpu))
        m.set_sequences([150, 150], [150, 150], [[0, 1, 2, 3], [4, 5, 6, 7]])
        outs.append(m.run().clone())
        m.H[:2].copy_(T["H"][:2].to(gpu))
        m.set_sequences([1, 1], [151, 151])
        outs.append(m.run()[:2].clone())
    for a, b in ((outs[0], outs[2]), (outs[1], outs[3])):
        assert rel_f(np_bits(a), np_bits(b)) <= 2.0 ** -4


# ------------------------------------------------------------------ weights that change under a captured graph
def test_captured_step_follows_its_weights(gpu):
    """set_weights between replays, of new tensors that do not stay: the graph reads the new
    weights, biases and gain and writes the gradients that the block shows."""
    rows, d, ffn = 40, 256, 768
    block, w, h, dout = gpt(gpu, rows, d, ffn, F.ACT_GELU, 11)
    eager = gpt(gpu, rows, d, ffn, F.ACT_GELU, 11)[0]

    def step():
        block.forward(h)
        block.backward(dout)

    step()
    block.capture(step)
    for turn in range(3):
        new = {k: (v.to(gpu) * (1.5 + turn)).to(v.dtype) for k, v in w.items()}
        block.set_weights(**new)
        del new
        junk = [torch.full((n,), 7.0, dtype=BF, device=gpu) for n in (d, ffn) for _ in range(8)]
        block.replay()
        eager.set_weights(**{k: (v.to(gpu) * (1.5 + turn)).to(v.dtype) for k, v in w.items()})
        eager.forward(h)
        eager.backward(dout)
        for name in ("out", "dh", "dw1", "dw2", "db1", "db2", "dg", "db"):
            assert torch.equal(getattr(block, name), getattr(eager, name)), (turn, name)
        assert all(bool((t == 7).all()) for t in junk)
    with pytest.raises(TypeError):
        block.set_weights(**{k: v.to(gpu).float() if k == "b1" else v.to(gpu) for k, v in w.items()})


def test_a_block_does_not_train_on_its_own_output(gpu):
    """forward(out) would overwrite what backward reads."""
    block, _, h, _ = gpt(gpu, 4, 64, 128, F.ACT_GELU, 1)
    with pytest.raises(ValueError, match="own output"):
        block.forward(block.forward(h))
    infer = gpt(gpu, 4, 64, 128, F.ACT_GELU, 1, train=False)[0]
    out = infer.forward(h).clone()
    want = infer.forward(out).clone()
    infer.forward(h)
    assert torch.equal(infer.forward(infer.out), want)
