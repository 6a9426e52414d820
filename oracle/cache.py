"""CPU oracle for the paged key/value cache of the decoder layer.

TEST INFRASTRUCTURE ONLY: plain, slow statements in fp64 of what the cache
calls of the library compute.  Rows cu_rows[s] <= r < cu_rows[s + 1] of a call
are the last tokens of sequence s, up to kv_len[s]; pages[s][i] holds its
positions i * page_size ..; a page number outside the cache, and every position
outside the table, is absent.

Codes: one bias per token and head from the largest magnitude (Sec. 2.3 Eq. 3),
cast with it (Sec. 2.1 Eq. 1), by the main oracle; the bias is kept as the
exponent byte 127 - b, for which b is clamped to 126.
"""
from __future__ import annotations

import numpy as np

from . import BF16, E4M3, E5M2, cast, decode_table, scale_bias  # noqa: F401
from .decoder import bf16_to_f64, round_bf16

CACHE_BF16 = 16
BLOCK = 16


class Cache:
    """Host copy of a cache: k [P, H, S, D], v [P, H, S / 16, D, 16] (uint8 codes
    or uint16 bf16 patterns), k_exp and v_exp [P, H, S]."""

    def __init__(self, k, v, k_exp, v_exp, fmt):
        self.k, self.v, self.k_exp, self.v_exp, self.fmt = k, v, k_exp, v_exp, fmt
        self.n_pages, self.heads, self.page_size, self.d_head = k.shape

    def copy(self):
        c = lambda a: None if a is None else a.copy()  # noqa: E731
        return Cache(c(self.k), c(self.v), c(self.k_exp), c(self.v_exp), self.fmt)

    def value(self, page, slot):
        """(k, v) fp64 [H, D] of one token."""
        k, v = self.k[page, :, slot], self.v[page, :, slot // BLOCK, :, slot % BLOCK]
        if self.fmt == CACHE_BF16:
            return bf16_to_f64(k), bf16_to_f64(v)
        tab = decode_table(self.fmt)
        ke, ve = self.k_exp[page, :, slot].astype(int) - 127, self.v_exp[page, :, slot].astype(int) - 127
        return tab[k] * np.ldexp(1.0, ke)[:, None], tab[v] * np.ldexp(1.0, ve)[:, None]


def place(cache, pages, s, pos):
    """(page, slot) of position pos of sequence s, None if absent."""
    i, slot = divmod(int(pos), cache.page_size)
    if pos < 0 or i >= pages.shape[1]:
        return None
    g = int(pages[s][i])
    return (g, slot) if 0 <= g < cache.n_pages else None


def tokens(cu, kv_len):
    """(row, sequence, position) of the rows of every sequence."""
    for s in range(len(kv_len)):
        n = int(cu[s + 1]) - int(cu[s])
        for i in range(n):
            yield int(cu[s]) + i, s, int(kv_len[s]) - n + i


def rotate(x, cs):
    """x [heads, D] fp64, cs [D / 2, 2]: (cos, sin) of the token's position."""
    half = x.shape[1] // 2
    a, b = x[:, :half], x[:, half:]
    c, s = cs[:, 0].astype(np.float64), cs[:, 1].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], axis=1)


def codes(x, fmt):
    """x [heads, D] float32: codes and exponent bytes."""
    q, e = np.empty(x.shape, dtype=np.uint8), np.empty(x.shape[0], dtype=np.uint8)
    for h in range(x.shape[0]):
        b = min(scale_bias(x[h], fmt)[0], 126)
        q[h], e[h] = cast(x[h], fmt, b), 127 - b
    return q, e


def append(qkv, cache, cu, kv_len, pages, n_heads, table):
    """qkv: bf16 patterns [rows, (n_heads + 2 H) D]; table [positions, D / 2, 2]
    float32 or None.  Writes into cache; returns q bf16 patterns (rows of no
    sequence: 0)."""
    nk, d = cache.heads, cache.d_head
    q = np.zeros((qkv.shape[0], n_heads * d), dtype=np.uint16)
    for r, s, pos in tokens(cu, kv_len):
        at = place(cache, pages, s, pos)
        if at is None:
            continue
        x = bf16_to_f64(qkv[r]).reshape(n_heads + 2 * nk, d)
        y = x[:n_heads + nk]
        if table is not None:
            y = rotate(y, table[pos])
        y = y.astype(np.float32)
        q[r] = round_bf16(y[:n_heads].astype(np.float64)).reshape(-1)
        g, slot = at
        k, v = y[n_heads:], x[n_heads + nk:].astype(np.float32)
        if cache.fmt == CACHE_BF16:
            cache.k[g, :, slot] = round_bf16(k.astype(np.float64))
            cache.v[g, :, slot // BLOCK, :, slot % BLOCK] = qkv[r].reshape(-1, d)[n_heads + nk:]
        else:
            cache.k[g, :, slot], cache.k_exp[g, :, slot] = codes(k, cache.fmt)
            cache.v[g, :, slot // BLOCK, :, slot % BLOCK], cache.v_exp[g, :, slot] = codes(v, cache.fmt)
    return q


def read(cache, cu, kv_len, pages, rows):
    """(k, v) bf16 patterns [rows, H D] (absent positions and rows of no sequence: 0)."""
    k = np.zeros((rows, cache.heads * cache.d_head), dtype=np.uint16)
    v = k.copy()
    for r, s, pos in tokens(cu, kv_len):
        at = place(cache, pages, s, pos)
        if at is not None:
            a, b = cache.value(*at)
            k[r], v[r] = round_bf16(a.reshape(-1)), round_bf16(b.reshape(-1))
    return k, v


def attention(q, cache, cu, kv_len, pages, n_heads, max_rows=None, window=0):
    """q bf16 patterns [rows, n_heads D].  Returns fp64 (o, a, t), [rows, n_heads D]
    the first two, [rows, n_heads] the last: the attention, the softmax-weighted
    mean of |v|, and over the keys a row sees the largest sum_d |q_d k_d| /
    sqrt(D) (what the roundings of the probabilities and scores scale with)."""
    nk, d = cache.heads, cache.d_head
    grp = n_heads // nk
    o = np.zeros((q.shape[0], n_heads, d))
    mean, top = np.zeros_like(o), np.zeros(o.shape[:2])
    for s in range(len(kv_len)):
        n = int(cu[s + 1]) - int(cu[s])
        if n == 0:
            continue
        longest = min(max(int(kv_len[s]), 0), pages.shape[1] * cache.page_size)
        at = [place(cache, pages, s, p) for p in range(longest)]
        present = np.array([a is not None for a in at], dtype=bool)
        K, V = np.zeros((longest, nk, d)), np.zeros((longest, nk, d))
        for p, a in enumerate(at):
            if a is not None:
                K[p], V[p] = cache.value(*a)
        for i in range(n if max_rows is None else min(n, max_rows)):
            pos = int(kv_len[s]) - n + i
            see = np.flatnonzero(present & (np.arange(longest) <= pos)
                                 & ((np.arange(longest) > pos - window) if window else True))
            if not len(see):
                continue
            r = int(cu[s]) + i
            qv = bf16_to_f64(q[r]).reshape(nk, grp, d)
            for hk in range(nk):
                k, v = K[see, hk], V[see, hk]
                sc = qv[hk] @ k.T / np.sqrt(d)
                p = np.exp(sc - sc.max(axis=1, keepdims=True))
                p /= p.sum(axis=1, keepdims=True)
                sl = slice(hk * grp, (hk + 1) * grp)
                o[r, sl], mean[r, sl] = p @ v, p @ np.abs(v)
                top[r, sl] = (np.abs(qv[hk]) @ np.abs(k).T).max(axis=1) / np.sqrt(d)
    return o.reshape(q.shape), mean.reshape(q.shape), top
