"""Infinities and NaN among cached keys and values reach the rows that see them, and only
those: every format, heads of 64 and 128, windows, key ranges and shares."""
import numpy as np
import pytest
import torch

from cache_cases import Case, blank, rand_bits, strided
from oracle import cache as C
from oracle import decoder as D
from paper_2309_17224_amd import fp8lin as F
from parity_util import np_bits
from test_gpu_cache import say

pytestmark = pytest.mark.gpu

E4, E5, BF = F.E4M3, F.E5M2, F.CACHE_BF16
INF, NAN = np.inf, np.nan
# patterns and what they are
PATTERNS = {E4: [(0x7F, NAN), (0xFF, NAN)],
            E5: [(0x7C, INF), (0xFC, -INF), (0x7D, NAN), (0x7F, NAN), (0xFE, NAN)],
            BF: [(0x7F80, INF), (0xFF80, -INF), (0x7F81, NAN), (0xFFFF, NAN)]}

#       new total at window capacity (pages of 64)
PLACES = [([40], [150], [140, 120], 0, None), ([5], [100], [97, 99], 0, None), ([70], [500], [400, 480], 65, None),
          ([5], [300], [232, 297], 65, None), ([90], [2500], [2430, 2470], 0, None),       # several key ranges
          ([90], [2500], [2300, 2301], 130, None), ([1, 1], [900, 70], [33, 833], 0, None),
          ([2], [9000], [8999, 8000], 0, 300),                                             # parts
          ([2] * 20, [900] * 20, [899, 600], 0, 900)]                                      # shares


@pytest.mark.parametrize("new,total,at,window,capacity", PLACES)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("fmt", [E4, E5, BF])
def test_values(gpu, fmt, dh, new, total, at, window, capacity):
    """Each pattern in a column of its own of two tokens; infinities of both signs in one column."""
    say("nonfinite values", fmt, dh, new[:3], total[:3], at, window, capacity)
    c = Case(86, 4, 2, dh, fmt, 64, new, total, capacity=capacity)
    q = rand_bits(c.rng, (c.rows, 4 * dh))
    cache, seqs = c.device(gpu)

    def out():
        o = blank(c.rows, 4 * dh, gpu)
        F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows, window=window, o=o)
        return np_bits(o).copy()

    clean = out()
    pos = np.arange(total[0] - new[0], total[0])
    sees = [(pos >= a) & ((pos - window < a) if window else True) for a in at]
    want = D.bf16_to_f64(clean).reshape(c.rows, 4, dh)
    seen = np.zeros(want.shape, dtype=bool)
    bits = cache.v.view(torch.int16 if fmt == BF else torch.uint8)
    pats = PATTERNS[fmt]

    def put(a, col, pattern):
        g, slot = C.place(c.host, c.pages, 0, at[a])
        bits[g, 1, slot // 16, col, slot % 16] = pattern - (0x10000 if fmt == BF and pattern > 0x7FFF else 0)

    def expect(rows, col, value):       # value heads of key/value head 1
        for r in np.flatnonzero(rows):
            want[r, 2:, col] = value
            seen[r, 2:, col] = True

    for i, (p, x) in enumerate(pats):
        col = 3 + 11 * i
        put(i % 2, col, p)
        expect(sees[i % 2], col, x)
    if fmt != E4:                       # +inf of one token, -inf of the other
        put(0, dh - 2, pats[0][0])
        put(1, dh - 2, pats[1][0])
        expect(sees[0], dh - 2, INF)
        expect(sees[1], dh - 2, -INF)
        expect(sees[0] & sees[1], dh - 2, NAN)
    got = out()
    assert seen.any()
    same = ~seen.reshape(c.rows, -1)
    assert np.array_equal(got[same], clean[same])
    f = D.bf16_to_f64(got).reshape(want.shape)
    assert np.array_equal(f[seen], want[seen], equal_nan=True)


@pytest.mark.parametrize("new,total,at,window,capacity", PLACES)
@pytest.mark.parametrize("fmt", [E4, E5, BF])
def test_keys(gpu, fmt, new, total, at, window, capacity):
    """A NaN in a key: NaN in every column of the heads of the rows that see it."""
    say("nan keys", fmt, new[:3], total[:3], at, window, capacity)
    for pattern, x in PATTERNS[fmt]:
        if not np.isnan(x):
            continue
        c = Case(87, 4, 2, 64, fmt, 64, new, total, capacity=capacity)
        q = rand_bits(c.rng, (c.rows, 256))
        cache, seqs = c.device(gpu)

        def out():
            o = blank(c.rows, 256, gpu)
            F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows, window=window, o=o)
            return np_bits(o).copy()

        clean = out()
        g, slot = C.place(c.host, c.pages, 0, at[0])
        cache.k.view(torch.int16 if fmt == BF else torch.uint8)[g, 1, slot, 9] = \
            pattern - (0x10000 if fmt == BF and pattern > 0x7FFF else 0)
        got = out()
        pos = np.arange(total[0] - new[0], total[0])
        nan = np.zeros(got.shape, dtype=bool)
        nan[:new[0], 128:] = ((pos >= at[0]) & ((pos - window < at[0]) if window else True))[:, None]
        assert nan.any() and np.array_equal(got[~nan], clean[~nan])
        assert ((got & 0x7FFF) > 0x7F80)[nan].all()
