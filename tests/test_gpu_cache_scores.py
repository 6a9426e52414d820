"""The cache attention with scores far beyond what an exponential takes: the weights
follow the differences of a row's scores, whatever the scores are.

All scores here are exact in fp32 (sums of products that share a grid), and so are
their differences, so that the bars do not grow with the scores:
  * a probability that is a difference's exponential: its product with log2(e) /
    sqrt(d_head) is off by 2^-23 of itself, the exponential by 2^-22: less than
    2^-15 for differences up to 2^7, beyond which a probability is 0;
  * from a product of the score and one of the maximum, whose products are up to 2^14
    (larger ones take the difference): the product of the maximum is rounded by 2^-11
    at most, and a row has two maxima in turn: 2^-10 in the exponent, 2^-10 of the weight;
  * probabilities rounded to bf16: 2^-8, sums of n: n 2^-23, output rounded: 2^-8.
"""
import numpy as np
import pytest
import torch

from cache_cases import Case, blank, strided
from oracle import cache as C
from oracle import decoder as D
from paper_2309_17224_amd import fp8lin as F
from parity_util import np_bits
from test_gpu_cache import say

pytestmark = pytest.mark.gpu

E4, E5, BF = F.E4M3, F.E5M2, F.CACHE_BF16


def code(x, fmt):
    """Codes (or bf16 patterns) of values that the format holds."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == BF:
        return C.round_bf16(x)
    tab = C.decode_table(fmt)
    at = np.argsort(tab[:0x78 if fmt == E5 else 0x7F])
    c = at[np.searchsorted(tab[at], x.ravel())].reshape(x.shape).astype(np.uint8)
    assert np.array_equal(tab[c], x)
    return c


def keys_of(c, dims):
    """The cache's keys: these values (of shape k[..., 0]) in the first dimensions, 0 in the others."""
    h = c.host
    h.k[...] = 0
    for i, x in enumerate(dims):
        h.k[..., i] = code(x, c.fmt)
    if h.k_exp is not None:
        h.k_exp[...] = 127


def compare(c, q, o, window=0):
    want, mean, _ = C.attention(q, c.host, c.cu, c.kv_len, c.pages, c.heads, window=window)
    got = D.bf16_to_f64(np_bits(o))
    n = int(c.kv_len.max())
    off = 1.02 * (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -15 + n * 2.0 ** -23) * mean
    lim = off + 2.0 ** -8 * (np.abs(want) + off)
    assert not (mean.reshape(-1, c.d_head).any(axis=1) & ~got.reshape(-1, c.d_head).any(axis=1)).any(), "a row of zeros"
    assert np.isfinite(got).all()
    worst = float((np.abs(got - want) / np.maximum(lim, 1e-30)).max())
    return worst


#       new total heads kv capacity window
SHAPES = [([40], [150], 4, 2, None, 0), ([90], [2500], 4, 2, None, 0), ([50], [300], 4, 2, 80, 0),
          ([40, 1], [150, 700], 4, 2, None, 0), ([70], [500], 8, 2, None, 90), ([1, 1], [900, 70], 4, 2, None, 0),
          ([1], [5000], 2, 2, None, 0)]


@pytest.mark.parametrize("new,total,heads,kv,capacity,window", SHAPES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("fmt", [E4, E5, BF])
def test_one_key_takes_all(gpu, fmt, dh, new, total, heads, kv, capacity, window):
    """Scores of 2^13 to 2^43 times every winning mantissa, rows of other maxima, signs and
    ordinary scores among them: the largest takes all, ties share."""
    say("one takes all", fmt, dh, new, total, heads, kv, capacity, window)
    c = Case(71, heads, kv, dh, fmt, 64, new, total, capacity=capacity)
    rng = c.rng
    worst = 0.0
    for top in (5.0, 6.0, 7.0) if fmt == E5 else (4.5, 5.0, 5.5, 6.0, 6.5, 7.0, 7.5):
        k0 = rng.integers(2, 9, c.host.k[..., 0].shape) / 2.0      # 1 to 4
        k0 = np.where(rng.random(k0.shape) < 0.02, top, k0)
        keys_of(c, [k0])
        cache, seqs = c.device(gpu)
        powers = (13, 17, 28, 31, 34, 36, 40, 43)
        for power in powers if max(total) < 300 else rng.choice(powers, 2, replace=False):
            power = int(power)
            q = np.zeros((c.rows, heads, dh))
            scale = rng.choice([1.0, 1.25, 1.5, 0.125, -1.0, 2.0 ** -power, 0.0], (c.rows, heads),
                               p=[0.4, 0.1, 0.1, 0.1, 0.1, 0.1, 0.1])
            q[:, :, 0] = scale * 2.0 ** power
            q = C.round_bf16(q.reshape(c.rows, -1))
            o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, heads, c.max_rows, window=window)
            w = compare(c, q, o, window)
            assert w <= 1.0, (top, power, w)
            worst = max(worst, w)
    print(f"worst {worst:.3f} of the bound", flush=True)


@pytest.mark.parametrize("new,total,heads,kv,capacity,window", SHAPES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("fmt", [E4, BF])
def test_differences_on_a_common_score(gpu, fmt, dh, new, total, heads, kv, capacity, window):
    """Scores that differ by ordinary amounts on top of a common +-2^10 to 2^22: many keys, then
    some whose probabilities are 2^8 times theirs, so that the maximum moves on the way."""
    say("common score", fmt, dh, new, total, heads, kv, capacity, window)
    c = Case(72, heads, kv, dh, fmt, 64, new, total, capacity=capacity)
    rng = c.rng
    late = rng.random(c.host.k[..., 0].shape) < 0.004
    # 256 and 1/64 to 3/64: with queries 2^(p - 8) and 64 * 64, scores of +-2^p + 64 .. 192
    keys_of(c, [np.full(late.shape, 256.0), np.where(late, rng.integers(2, 4, late.shape), 1) / 64.0])
    cache, seqs = c.device(gpu)
    worst = 0.0
    for power in (10, 14, 16, 17, 18, 20, 21, 22):
        for sign in (1.0, -1.0) if max(total) < 1000 else (rng.choice([1.0, -1.0]),):
            q = np.zeros((c.rows, heads, dh))
            q[:, :, 0] = sign * 2.0 ** (power - 8)
            q[:, :, 1] = 64.0 * 64.0
            q = C.round_bf16(q.reshape(c.rows, -1))
            o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, heads, c.max_rows, window=window)
            w = compare(c, q, o, window)
            print(power, sign, f"{w:.3f}", flush=True)
            assert w <= 1.0, (power, sign, w)
            worst = max(worst, w)
    print(f"worst {worst:.3f} of the bound", flush=True)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("fmt", [E4, BF])
def test_a_maximum_that_is_large_on_the_way_only(gpu, fmt, dh):
    """The first keys' scores are -4.5 to -7.5 times 2^24 to 2^43, the others' ordinary: the first
    have no weight, and the rounding of theirs leaves none."""
    say("large on the way", fmt, dh)
    for new, total in (([40], [150]), ([60, 1], [400, 300])):
        c = Case(74, 4, 2, dh, fmt, 64, new, total)
        for top in (4.5, 5.0, 6.5, 7.5):
            k0 = c.rng.integers(0, 3, c.host.k[..., 0].shape) / 2.0
            keys_of(c, [np.zeros_like(k0), k0])
            for s in range(len(new)):
                for pos in range(70):
                    page, slot = C.place(c.host, c.pages, s, pos)
                    c.host.k[page, :, slot, 0] = code(np.full(2, top), fmt)
            cache, seqs = c.device(gpu)
            for power in (24, 30, 35, 43):
                q = np.zeros((c.rows, 4, dh))
                q[:, :, 0] = -2.0 ** power
                q[:, :, 1] = 3.0
                q = C.round_bf16(q.reshape(c.rows, -1))
                o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows)
                assert compare(c, q, o) <= 1.0, (new, top, power)


def test_ordinary_rows_keep_their_bits_beside_large_scores(gpu):
    """Rows of ordinary scores in the tile of one whose scores are of 2^36: bits as without it."""
    say("ordinary beside large")
    for fmt in (E4, BF):
        c = Case(73, 4, 2, 128, fmt, 64, [60], [400])
        q = c.rng.standard_normal((60, 512)).astype(np.float32)
        q = C.round_bf16(q.astype(np.float64))
        cache, seqs = c.device(gpu)
        clean = np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 60)).copy()
        big = q.copy()
        big[17, 128:256] = C.round_bf16(2.0 ** 34 * c.rng.standard_normal(128))
        o = blank(60, 512, gpu)
        got = np_bits(F.llama_cache_attention(strided(big, gpu, 0), cache, seqs, 4, 60, o=o))
        torch.cuda.synchronize()
        same = np.ones((60, 512), dtype=bool)
        same[17, 128:256] = False
        assert np.array_equal(got[same], clean[same])
        row = D.bf16_to_f64(got[17, 128:256])
        assert np.isfinite(row).all() and row.any()
