"""Pins of the cache oracle (CPU): against the decoder oracle, the main oracle
and small hand-made cases."""
import numpy as np
import pytest

import oracle as orc_mod
from cache_cases import Case, rand_bits
from oracle import cache as C
from oracle import decoder as D

FMTS = [C.E4M3, C.E5M2, C.CACHE_BF16]


@pytest.mark.parametrize("fmt", FMTS)
def test_append_then_read_gives_the_quantised_values(fmt):
    c = Case(1, 4, 2, 64, fmt, 16, [5, 1, 17], [5, 30, 40])
    qkv = rand_bits(c.rng, (c.rows, 8 * 64))
    q = C.append(qkv, c.host, c.cu, c.kv_len, c.pages, 4, None)
    assert np.array_equal(q, qkv[:, :4 * 64])                 # no table: unrotated
    k, v = C.read(c.host, c.cu, c.kv_len, c.pages, c.rows)
    for got, want in ((k, qkv[:, 4 * 64:6 * 64]), (v, qkv[:, 6 * 64:])):
        g, w = D.bf16_to_f64(got), D.bf16_to_f64(want)
        if fmt == C.CACHE_BF16:
            assert np.array_equal(got, want)
            continue
        for r in range(c.rows):
            for h in range(2):
                x = want[r, h * 64:(h + 1) * 64]
                b = orc_mod.scale_bias(x, fmt)[0]
                ref = orc_mod.decode_table(fmt)[orc_mod.cast(x, fmt, b)] * 2.0 ** -b
                assert np.array_equal(g[r, h * 64:(h + 1) * 64], ref)
        assert np.max(np.abs(g - w)) <= 2.0 ** -3 * np.max(np.abs(w))


def test_prefill_through_a_bf16_cache_equals_the_decoder_oracle():
    n, heads, nk, d = 40, 4, 2, 128
    c = Case(2, heads, nk, d, C.CACHE_BF16, 16, [n], [n])
    qkv = rand_bits(c.rng, (n, (heads + 2 * nk) * d))
    pos = np.arange(c.max_pages * 16)[:, None] * 10000.0 ** (-2.0 * np.arange(d // 2) / d)
    table = np.stack([np.cos(pos), np.sin(pos)], axis=2).astype(np.float32)
    q = C.append(qkv, c.host, c.cu, c.kv_len, c.pages, heads, table)
    rot = D.rope(qkv[:, :(heads + nk) * d], n, d)
    same = q == rot[:, :heads * d]
    assert same.mean() > 0.999       # the table is rounded to fp32
    k, v = C.read(c.host, c.cu, c.kv_len, c.pages, n)
    o, mean, top = C.attention(q, c.host, c.cu, c.kv_len, c.pages, heads)
    assert np.array_equal(D.round_bf16(o), D.attention(q, k, v, n, heads, nk, d))
    assert np.all(np.abs(o) <= mean + 1e-12) and np.all(top > 0)


def test_a_chunk_sees_what_the_whole_sees():
    c = Case(3, 2, 1, 64, C.E4M3, 32, [21], [77])
    q = rand_bits(c.rng, (21, 128))
    o = C.attention(q, c.host, c.cu, c.kv_len, c.pages, 2)[0]
    for i in (0, 7, 20):     # token by token
        o1 = C.attention(q[i:i + 1], c.host, [0, 1], [77 - 20 + i], c.pages, 2)[0]
        assert np.allclose(o1[0], o[i], rtol=0, atol=1e-13)


def test_absent_places_and_empty_rows():
    c = Case(4, 2, 2, 64, C.E5M2, 16, [4, 3], [2, 40])
    q = rand_bits(c.rng, (7, 128))
    c.pages[1, 0] = -1                       # an absent page
    o = C.attention(q, c.host, c.cu, c.kv_len, c.pages, 2, window=5)[0]
    assert not o[:2].any() and o[2:4].any()  # positions -2, -1, then 0, 1
    w = C.attention(q[4:], c.host, [0, 3], [40], c.pages[1:], 2, window=5)[0]
    assert np.array_equal(w, o[4:])
    c.pages[1] = -1
    o = C.attention(q, c.host, c.cu, c.kv_len, c.pages, 2)[0]
    assert not o[4:].any()
    assert not C.read(c.host, c.cu, c.kv_len, c.pages, 7)[0][4:].any()
    before = c.host.copy()
    assert not C.append(rand_bits(c.rng, (7, 6 * 64)), c.host, c.cu, c.kv_len, c.pages, 2, None)[4:].any()
    assert (c.host.k != before.k).any(axis=(1, 2, 3)).sum() <= 1


def test_one_key_returns_its_value():
    c = Case(5, 4, 4, 64, C.E4M3, 16, [1], [1])
    o = C.attention(rand_bits(c.rng, (1, 256)), c.host, c.cu, c.kv_len, c.pages, 4)[0]
    assert np.array_equal(o.reshape(4, 64), c.host.value(c.pages[0, 0], 0)[1])
