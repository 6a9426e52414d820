"""The decoder layer over a paged key/value cache: the append, the attention with
its fused quantise and the layer's other calls together, as a serving loop makes
them.

Bars: the cache holds what the oracle appends from the layer's own QKV output,
bit for bit; the attention is within the bound of the attention tests of the
oracle's over that cache; its codes are fp8_quantise's of its bf16 output.  Over
an unquantised cache the whole layer agrees with the layer that attends within a
call: the attention within rel_F 1e-2 (two roundings of probabilities and
outputs), what follows within half an E4M3 step, 2^-4, the agreement of FP8 chains
whose inputs differ by bf16 roundings (a value that lies at a border moves by a
whole step).  Captured calls equal eager ones bit for bit.
"""
import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import decoder as D
from paper_2309_17224_amd import decoder as DL
from paper_2309_17224_amd import fp8lin as F
from paper_2309_17224_amd import workloads as wl
from parity_util import np_bits, rel_f
from test_gpu_cache import bound

pytestmark = pytest.mark.gpu

FP8_CHAIN = 2.0 ** -4


def config(rows, seq_len=150, heads=8, kv=2):
    return wl.LayerConfig("cached-layer", 9, "small layer over a cache", 512, heads, kv, 128, 1408, rows, seq_len, 0.05)


def weights(cfg, dev):
    return {t.name: wl.make_layer_tensor(cfg, t.name).to(dev) for t in cfg.tensors() if t.name != "H"}


def hidden(rows, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((rows, 512), generator=g).to(torch.bfloat16)


class Shadow:
    """The oracle's copy of a layer's cache, appended to call by call."""

    def __init__(self, layer):
        k = layer.cache
        h = [None if t is None else np_bits(t).copy() for t in (k.k, k.v, k.k_exp, k.v_exp)]
        self.cache = C.Cache(*h, k.fmt)
        self.c = layer.cfg
        self.table = layer.table.cpu().numpy().reshape(-1, 64, 2)
        self.heads, self.d_head = layer.cfg.n_heads, 128

    def check(self, layer, raw_qkv):
        cu, kv, pages = (t.cpu().numpy() for t in (layer.seqs.cu_rows, layer.seqs.kv_len, layer.seqs.pages))
        n, dq = int(cu[-1]), self.c.n_heads * 128
        q = C.append(raw_qkv, self.cache, cu, kv, pages, self.c.n_heads, self.table)
        assert np.array_equal(np_bits(layer.qkv)[:n, :dq], q[:n])
        for name in ("k", "v", "k_exp", "v_exp"):
            ref = getattr(self.cache, name)
            assert ref is None or np.array_equal(np_bits(getattr(layer.cache, name)), ref), name
        want, mean, top = C.attention(q, self.cache, cu, kv, pages, self.c.n_heads, window=layer.window)
        self.kv_len = kv
        got = D.bf16_to_f64(np_bits(layer.att.x))
        worst = (np.abs(got - want)[:n] / bound(self, want, mean, top)[:n]).max()
        print("attention: worst %.3f of the bound" % worst, flush=True)
        assert worst <= 1.0
        # the quantise's bias is of the live rows; the layer's padding rows hold zeros
        q8, _, b, a, fl = F.fp8_quantise(layer.att.x, F.E4M3)
        assert torch.equal(layer.att.q, q8) and layer.att.scal.cpu().tolist() == [int(b), int(a), int(fl)]


def run_checked(layer, shadow, H):
    layer.H[:H.shape[0]] = H
    for label, _, _, fn in layer.calls:
        if label.startswith("rope"):
            torch.cuda.synchronize()
            raw = np_bits(layer.qkv).copy()
        fn()
        if label.startswith("cache attention"):
            torch.cuda.synchronize()
            shadow.check(layer, raw)
    return layer.out


@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2, F.CACHE_BF16])
def test_serving_loop(gpu, fmt):
    """Prefill chunks of odd lengths, then single tokens, sequences joining and
    leaving, padding rows, through one layer object."""
    print("\n[case] serving loop", fmt, flush=True)
    cfg = config(48)
    layer = DL.CachedDecoderLayer(cfg, weights(cfg, gpu), gpu, n_seqs=3, max_pages=6, page_size=16, n_pages=20,
                                  kv_fmt=fmt)
    layer.cache.k.view(torch.uint8).fill_(0x7F)       # NaN where nothing has been written
    layer.cache.v.view(torch.uint8).fill_(0x7F)
    if layer.cache.k_exp is not None:
        layer.cache.k_exp.fill_(255)
        layer.cache.v_exp.fill_(255)
    shadow = Shadow(layer)
    pages = [[3, 11, 7, 0, 19, 5], [1, 2, 18], [4, 17, 6, 9]]
    length = [0, 0, 0]
    for step, rows in enumerate([[37, 0, 0], [11, 20, 0], [1, 13, 34], [1, 1, 1], [0, 1, 1], [1, 0, 2], [1, 1, 1]]):
        length = [a + b for a, b in zip(length, rows)]
        layer.set_sequences(rows, length, pages)
        out = run_checked(layer, shadow, hidden(sum(rows), 100 + step).to(gpu))
        torch.cuda.synchronize()
        assert torch.isfinite(out.float()).all()


def test_matches_the_layer_without_a_cache(gpu):
    """Two sequences of 150 tokens, whole and in chunks, over a bf16 cache."""
    print("\n[case] against the layer without a cache", flush=True)
    cfg = config(300)
    W = weights(cfg, gpu)
    H = hidden(300, 7).to(gpu)
    plain = DL.DecoderLayer(cfg, W, gpu)
    plain.H.copy_(H)
    ref = plain.run().clone()
    whole = DL.CachedDecoderLayer(cfg, W, gpu, n_seqs=2, max_pages=10, page_size=16, kv_fmt=F.CACHE_BF16)
    pages = [[2 * i for i in range(10)], [2 * i + 1 for i in range(10)]]
    whole.set_sequences([150, 150], [150, 150], pages)
    whole.H.copy_(H)
    whole.run()
    torch.cuda.synchronize()
    e = rel_f(np_bits(whole.att.x), np_bits(plain.att.x)), rel_f(np_bits(whole.out), np_bits(ref))
    print("whole: attention %.2e, out %.2e" % e, flush=True)
    assert e[0] <= 1e-2 and e[1] <= FP8_CHAIN
    part = config(64)
    chunked = DL.CachedDecoderLayer(part, W, gpu, n_seqs=2, max_pages=10, page_size=16, kv_fmt=F.CACHE_BF16)
    done, got = [0, 0], torch.zeros_like(ref)
    for rows in ([50, 14], [64, 0], [30, 34], [6, 50], [0, 52]):
        done = [a + b for a, b in zip(done, rows)]
        chunked.set_sequences(rows, done, pages)
        src = [torch.arange(150 * s + done[s] - rows[s], 150 * s + done[s]) for s in (0, 1)]
        at = torch.cat(src).to(gpu)
        chunked.H[:len(at)] = H[at]
        chunked.run()
        got[at] = chunked.out[:len(at)]
    torch.cuda.synchronize()
    assert done == [150, 150]
    e = rel_f(np_bits(got), np_bits(ref))
    print("in chunks: out %.2e" % e, flush=True)
    assert e <= FP8_CHAIN


def test_captured_decode(gpu):
    """A step of three sequences captured once, replayed token by token; two layers
    captured over the same cache of pages and the same lengths."""
    print("\n[case] captured decode", flush=True)
    cfg = config(4)
    W = weights(cfg, gpu)
    pages = [[0, 4, 5, 9], [1, 2, 8, 3], [6, 7, 11, 10]]

    def fresh():
        layer = DL.CachedDecoderLayer(cfg, W, gpu, n_seqs=3, max_pages=4, page_size=32, kv_fmt=F.E4M3, max_rows=1)
        for t in (layer.cache.k, layer.cache.v, layer.cache.k_exp, layer.cache.v_exp):
            g = torch.Generator(device=gpu).manual_seed(5)
            t.copy_(torch.randint(100, 126, t.shape, generator=g, device=gpu, dtype=torch.int32).to(torch.uint8))
        layer.set_sequences([1, 1, 1], [40, 7, 101], pages)
        layer.H.copy_(hidden(4, 3).to(gpu))
        return layer

    eager, cap = fresh(), fresh()
    eager.run()
    cap.run()
    cap.capture()
    eager.run()
    cap.replay()
    for t in range(5):
        H = hidden(4, 50 + t).to(gpu)
        for layer in (eager, cap):
            layer.H.copy_(H)
            layer.set_sequences([1, 1, 1] if t != 2 else [1, 0, 1], [41 + t, 8 + t, 102 + t])
        eager.run()
        cap.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.out, cap.out) and torch.equal(eager.att.q, cap.att.q)
        assert torch.equal(eager.cache.k, cap.cache.k) and torch.equal(eager.cache.v, cap.cache.v)


def test_set_sequences_refuses(gpu):
    print("\n[case] refusals", flush=True)
    cfg = config(4)
    layer = DL.CachedDecoderLayer(cfg, weights(cfg, gpu), gpu, n_seqs=2, max_pages=2, page_size=16, max_rows=3)
    for rows, kv in (([1], [1, 2]), ([1, 1, 1], [1, 1, 1]), ([4], [4]), ([3, 2], [3, 2]), ([-1], [1]), ([2], [1]),
                     ([1], [33])):
        with pytest.raises(ValueError):
            layer.set_sequences(rows, kv)
    for pages in ([[0], [1], [2]], [[0, 1, 2]]):
        with pytest.raises(ValueError):
            layer.set_sequences([1], [1], pages)
    other = F.KVCache(4, 4, 128, 16, F.E4M3, gpu)
    with pytest.raises(ValueError):
        DL.CachedDecoderLayer(cfg, weights(cfg, gpu), gpu, n_seqs=2, max_pages=2, cache=other)
    layer.set_sequences([3], [32], [[0, 1]])
