"""Exponent bytes that no append writes: 255 counts as 254 in every call, and where a row
does not see its token it does not reach the row; 0 is 2^-127.  And values at both ends of
the range that the attention takes."""
import numpy as np
import pytest
import torch

from cache_cases import Case, blank, rand_bits, strided
from oracle import cache as C
from oracle import decoder as D
from paper_2309_17224_amd import fp8lin as F
from parity_util import np_bits
from test_gpu_cache import bound, check, say

pytestmark = pytest.mark.gpu

E4, E5, BF = F.E4M3, F.E5M2, F.CACHE_BF16

#       new total at window: rows at the token's place or behind it, and within the window, see it
TOKENS = [([40], [150], 140, 0), ([5], [100], 97, 0), ([70], [500], 400, 65), ([5], [300], 232, 65),
          ([90], [2500], 2430, 0), ([70, 1], [70, 900], 33, 0), ([1], [700], 640, 0)]


@pytest.mark.parametrize("new,total,at,window", TOKENS)
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("dh", [64, 128])
def test_255_stays_where_it_is_seen(gpu, dh, fmt, new, total, at, window):
    """Rows that do not see the token keep their bits; those that do are as with 254."""
    say("exponent 255", dh, fmt, new, total, at, window)
    for where in ("v_exp", "k_exp", "both"):
        c = Case(81, 4, 2, dh, fmt, 16, new, total)
        q = rand_bits(c.rng, (c.rows, 4 * dh))
        cache, seqs = c.device(gpu)
        g, slot = C.place(c.host, c.pages, 0, at)

        def out():
            o = blank(c.rows, 4 * dh, gpu)
            F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows, window=window, o=o)
            return np_bits(o).copy()

        clean, got = out(), []
        for e in (254, 255):
            for name in ("v_exp", "k_exp"):
                if where in (name, "both"):
                    getattr(cache, name)[g, 1, slot] = e
            got.append(out())
        pos = np.arange(total[0] - new[0], total[0])
        sees = np.zeros(c.rows, dtype=bool)
        sees[:new[0]] = (pos >= at) & ((pos - window < at) if window else True)
        assert np.array_equal(got[1][~sees], clean[~sees]), where
        assert np.array_equal(got[1][:, :2 * dh], clean[:, :2 * dh]), where      # the other key/value head
        assert np.array_equal(got[1], got[0]), where


@pytest.mark.parametrize("new,total,at,window", TOKENS)
@pytest.mark.parametrize("fmt", [E4, E5])
def test_255_is_254(gpu, fmt, new, total, at, window):
    """A token of one tiny value, keys of 0: the oracle's result with 254."""
    say("255 is 254", fmt, new, total, at, window)
    c = Case(82, 4, 2, 128, fmt, 16, new, total)
    g, slot = C.place(c.host, c.pages, 0, at)
    c.host.k[g, 1, slot] = 0
    c.host.v[g, 1, slot // 16, :, slot % 16] = 0
    c.host.v[g, 1, slot // 16, 7, slot % 16] = 0x81        # the smallest, negative
    c.host.k_exp[g, 1, slot] = c.host.v_exp[g, 1, slot] = 255
    q = rand_bits(c.rng, (c.rows, 512))
    cache, seqs = c.device(gpu)
    c.host.k_exp[g, 1, slot] = c.host.v_exp[g, 1, slot] = 254
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows, window=window)
    check(c, q, o, window)


@pytest.mark.parametrize("fmt", [E4, E5])
def test_read_of_every_exponent(gpu, fmt):
    """Codes times 2^(exp - 127), 255 as 254; what bf16 does not hold becomes infinite."""
    say("read of every exponent", fmt)
    c = Case(83, 2, 2, 64, fmt, 16, [256], [256])
    for pos in range(256):
        g, slot = C.place(c.host, c.pages, 0, pos)
        c.host.k_exp[g, :, slot] = c.host.v_exp[g, :, slot] = pos
        c.host.k[g, :, slot, :8] = np.arange(8)
        c.host.v[g, :, slot // 16, :8, slot % 16] = np.arange(8)
    cache, seqs = c.device(gpu)
    k, v = F.llama_cache_read(cache, seqs, 256)
    torch.cuda.synchronize()
    for e in (c.host.k_exp, c.host.v_exp):
        e[e == 255] = 254
    with np.errstate(over="ignore"):
        wk, wv = C.read(c.host, c.cu, c.kv_len, c.pages, 256)
    assert np.array_equal(np_bits(k), wk) and np.array_equal(np_bits(v), wv)


@pytest.mark.parametrize("heads", [4, 64])
@pytest.mark.parametrize("fmt", [E4, E5])
def test_exponent_0(gpu, fmt, heads):
    """One token with exponents 0: its values, code * 2^-127, exactly (64 heads: 32 rows a head)."""
    say("exponent 0", fmt, heads)
    c = Case(84, heads, 2, 64, fmt, 16, [1], [1])
    c.host.k_exp[...] = c.host.v_exp[...] = 0
    c.host.v[c.host.v & 0x7F < 0x40] = 0x45                # bf16 holds them
    q = rand_bits(c.rng, (1, heads * 64))
    cache, seqs = c.device(gpu)
    o = D.bf16_to_f64(np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, heads, 1)))
    want = np.repeat(c.host.value(c.pages[0, 0], 0)[1], heads // 2, axis=0).reshape(1, -1)
    assert np.array_equal(o, want)


@pytest.mark.parametrize("new,total,at,window", TOKENS)
@pytest.mark.parametrize("fmt", [E4, E5, BF])
@pytest.mark.parametrize("large", [True, False])
def test_range_of_values(gpu, large, fmt, new, total, at, window):
    """The largest values whose sums are stated to be finite, of one sign, and small
    exponents: within the bound, there with 2^-134 of the largest code for each key."""
    say("range of values", large, fmt, new, total, window)
    c = Case(85, 4, 2, 128, fmt, 16, new, total)
    n = max(total)
    if fmt == BF:       # scaled by a power of two
        e = 120 - int(np.ceil(np.log2(n))) if large else -120
        v = np.abs(c.rng.standard_normal(c.host.v.shape)) if large else c.rng.standard_normal(c.host.v.shape)
        v = np.clip(v / 4, -0.996, 0.996)
        c.host.v[...] = C.round_bf16(np.ldexp(v, e))
        code = 2.0 ** e
    else:
        top = 8.81 if fmt == E4 else 15.81                 # log2 of the largest code, rounded up
        e = int(np.ceil(120 - np.log2(n) - top)) - 1 if large else -113
        c.host.v_exp[...] = c.rng.integers(e + 125, e + 128, c.host.v_exp.shape)
        if large:
            c.host.v[...] &= 0x7F
        code = 2.0 ** top
        assert not large or n * 2.0 ** (top + e) < 2.0 ** 120
    q = rand_bits(c.rng, (c.rows, 512), 2.0)
    cache, seqs = c.device(gpu)
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows, window=window)
    want, mean, top = C.attention(q, c.host, c.cu, c.kv_len, c.pages, 4, window=window)
    got = D.bf16_to_f64(np_bits(o))
    tiny = 0.0 if large else n * 2.0 ** -134 * code + 2.0 ** -134      # the output below bf16's normal range
    scale = 2.0 ** (-100 if large else 100)                # bound's own floor is for ordinary values
    lim = bound(c, want * scale, mean * scale, top) / scale + 1.02 * tiny
    assert np.isfinite(got).all()
    print("worst %.3f of the bound" % (np.abs(got - want) / lim).max(), flush=True)
    assert (np.abs(got - want) <= lim).all()
