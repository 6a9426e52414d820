"""Inputs of the paged key/value cache tests: sequences, page tables and caches
from a seed, on the host (numpy), and their device copies."""
from __future__ import annotations

import numpy as np
import torch

from oracle import cache as C
from paper_2309_17224_amd import fp8lin as F
from paper_2309_17224_amd import workloads as wl

SENTINEL = 0x4321   # bf16 pattern of outputs that a call must leave


def rand_bits(rng, shape, std=1.0):
    x = torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)
    return wl.bf16_bits(x)


class Case:
    """Sequences with `new` rows at the end of `total` tokens, `tail` rows behind
    the last one; pages in random order, unused entries of the table garbage."""

    def __init__(self, seed, heads, kv_heads, d_head, fmt, page, new, total, tail=0, spare=3, capacity=None):
        self.rng = rng = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.d_head, self.fmt, self.page = heads, kv_heads, d_head, fmt, page
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.kv_len = np.array(total, dtype=np.int32)
        self.rows, self.max_rows = int(self.cu[-1]) + tail, max(max(new), 1)
        need = [max(0, -(-t // page)) for t in total]
        self.max_pages = max(max(need), 1) + 1 if capacity is None else capacity
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages)
        self.pages = np.full((len(new), self.max_pages), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            n = min(n, self.max_pages)
            self.pages[s, :n] = order[at:at + n]
            at += n
        junk = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31], self.pages.shape)
        used = np.arange(self.max_pages)[None, :] < np.array(need)[:, None]
        self.pages = np.where(used, self.pages, junk).astype(np.int32)
        self.host = self._cache(n_pages)

    def _cache(self, P):
        rng, H, S, D = self.rng, self.kv_heads, self.page, self.d_head
        ks, vs, es = (P, H, S, D), (P, H, S // 16, D, 16), (P, H, S)
        if self.fmt == F.CACHE_BF16:
            return C.Cache(rand_bits(rng, ks, 1.5), rand_bits(rng, vs), None, None, self.fmt)
        # codes of every magnitude but NaN and infinities, exponents a few binades apart
        top = {F.E4M3: 0x7E, F.E5M2: 0x7B}[self.fmt]
        low = {F.E4M3: 0x28, F.E5M2: 0x34}[self.fmt]

        def codes(shape):
            c = rng.integers(low, top + 1, shape) | (rng.integers(0, 2, shape) << 7)
            return np.where(rng.random(shape) < 0.05, rng.integers(0, low, shape), c).astype(np.uint8)

        # largest codes 2^8 (E4M3), 2^15: scores of a few units, values of about one
        mid = 127 - (8 if self.fmt == F.E4M3 else 15)
        return C.Cache(codes(ks), codes(vs), rng.integers(mid - 2, mid + 1, es).astype(np.uint8),
                       rng.integers(mid - 2, mid + 1, es).astype(np.uint8), self.fmt)

    def poison_unused(self):
        """NaN codes (or bf16 NaNs) and exponent 255 in every slot that holds no
        token of a sequence."""
        h = self.host
        live = np.zeros((h.n_pages, self.page), dtype=bool)
        for s in range(len(self.kv_len)):
            for p in range(int(self.kv_len[s])):
                at = C.place(h, self.pages, s, p)
                if at is not None:
                    live[at] = True
        dead = ~live
        nan = 0x7FFF if self.fmt == F.CACHE_BF16 else 0x7F
        for p, t in zip(*np.nonzero(dead)):
            h.k[p, :, t] = nan
            h.v[p, :, t // 16, :, t % 16] = nan
            if h.k_exp is not None:
                h.k_exp[p, :, t] = 255
                h.v_exp[p, :, t] = 255

    # ---- device copies
    def device(self, dev):
        bf = self.fmt == F.CACHE_BF16

        def up(a):
            if a is None:
                return None
            t = torch.from_numpy(np.ascontiguousarray(a.view(np.int16) if bf else a)).to(dev)
            return t.view(torch.bfloat16) if bf else t

        h = self.host
        cache = F.KVCache(h.n_pages, self.kv_heads, self.d_head, self.page, self.fmt, dev, k=up(h.k), v=up(h.v),
                          k_exp=up(h.k_exp), v_exp=up(h.v_exp))
        i = lambda a: torch.from_numpy(a).to(dev)  # noqa: E731
        # rows of the page table apart from each other
        wide = torch.full((self.pages.shape[0], self.max_pages + 3), 7, dtype=torch.int32, device=dev)
        wide[:, :self.max_pages] = i(self.pages)
        return cache, F.CacheSeqs(i(self.cu), i(self.kv_len), wide[:, :self.max_pages])

    def table(self, dev):
        return F.llama_rope_table(self.max_pages * self.page, self.d_head, device=dev)


def strided(bits, dev, extra):
    """Device bf16 tensor of these patterns whose rows are `extra` elements apart."""
    rows, cols = bits.shape
    t = torch.full((rows, cols + extra), SENTINEL, dtype=torch.int16, device=dev)
    t[:, :cols] = torch.from_numpy(bits.view(np.int16)).to(dev)
    return t.view(torch.bfloat16)[:, :cols]


def blank(rows, cols, dev, extra=0):
    return torch.full((rows, cols + extra), SENTINEL, dtype=torch.int16, device=dev).view(torch.bfloat16)[:, :cols]
