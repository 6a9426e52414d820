"""The cache attention where its work is cut: equal shares over long ragged batches,
parts of one sequence, key ranges of chunks; and the workspace that carries it.

Which cut a call takes follows the capacity of its page table, not the lengths in
it, so that short sequences under a long table reach each of them.  Bars are those
of test_gpu_cache.py."""
import ctypes

import numpy as np
import pytest
import torch

from cache_cases import SENTINEL, Case, blank, rand_bits, strided
from oracle import cache as C
from oracle import decoder as D
from paper_2309_17224_amd import fp8lin as F
from parity_util import np_bits
from test_gpu_cache import bound, check, say

pytestmark = pytest.mark.gpu

E4, E5, BF = F.E4M3, F.E5M2, F.CACHE_BF16


def counts(ws):
    return int(ws[:F.CACHE_WS_COUNTS].count_nonzero())


def lens(seed, n, top, zero=0.1):
    rng = np.random.default_rng(seed)
    return [0 if rng.random() < zero else int(x) for x in rng.integers(1, top, n)]


#   heads kv dh fmt page capacity new total tail window
# items (sequences times key/value heads) times tiles of 64 keys of the table: 32768 at least
SHARES = [
    (16, 8, 128, E4, 1024, 48, [1] * 6, [1, 5000, 64, 0, 777, 9000], 2, 0),
    (16, 8, 128, E4, 1024, 48, [1] * 6, [40, 5000, 64, 0, 777, 9000], 0, 700),     # a window
    (4, 2, 128, E5, 16, 1000, [1] * 70, lens(1, 70, 600), 0, 0),                   # more sequences than lanes
    (4, 1, 64, BF, 128, 128, [1] * 150, lens(2, 150, 400), 3, 0),
    (2, 1, 64, E4, 64, 64, [1] * 1024, lens(3, 1024, 90), 0, 0),                   # as many sequences as are cut
    (2, 1, 64, E4, 64, 64, [1] * 1025, lens(4, 1025, 90), 0, 0),                   # one more
    (8, 4, 128, BF, 64, 256, [1] * 20 + [0] * 20 + [2], lens(5, 41, 900), 1, 0),   # absent ones, two tokens
    (4, 2, 128, E4, 1024, 300, [1] * 4, [0, 0, 0, 0], 0, 0),                       # no keys at all
    (4, 2, 128, E4, 1024, 300, [1] * 4, [1, 0, 0, 1], 0, 0),                       # shares without work
    (1, 1, 64, E4, 1024, 2048, [1], [20000], 0, 0),                                # one item
    (16, 4, 128, E4, 512, 30, [1] * 30 + [50, 1, 0, 5] + [1] * 6, lens(6, 40, 700), 2, 0),  # a chunk among them
    (4, 2, 128, E5, 256, 1030, [2, 8, 9, 1], [2, 40, 1200, 3000], 0, 0),            # 4, 16, 18 and 2 packed rows
]


@pytest.mark.parametrize("heads,kv,dh,fmt,page,capacity,new,total,tail,window", SHARES)
def test_shares(gpu, heads, kv, dh, fmt, page, capacity, new, total, tail, window):
    say("shares", heads, kv, dh, fmt, page, capacity, new[:4], total[:4], tail, window)
    c = Case(51, heads, kv, dh, fmt, page, new, total, tail, capacity=capacity)
    c.poison_unused()
    q = rand_bits(c.rng, (c.rows, heads * dh))
    cache, seqs = c.device(gpu)
    qd = strided(q, gpu, 0)
    ws = F.cache_attention_workspace(c.rows, heads, cache, seqs, c.max_rows)
    outs = []
    for _ in range(3):
        o = blank(c.rows, heads * dh, gpu)
        outs.append(F.llama_cache_attention(qd, cache, seqs, heads, c.max_rows, window=window, o=o, ws=ws))
    torch.cuda.synchronize()
    check(c, q, outs[0], window)
    assert counts(ws) == 0
    for o in outs[1:]:
        assert torch.equal(o.view(torch.int16), outs[0].view(torch.int16))
    # with the fused quantise
    live = int(c.cu[-1])
    rq, _, rb, ra, rf = F.fp8_quantise(outs[0][:live], E4)
    q8 = torch.full((c.rows, heads * dh), 0x55, dtype=torch.uint8, device=gpu)
    s = torch.zeros(3, dtype=torch.int32, device=gpu)
    for pred in (None, int(rb.item()), int(rb.item()) + 2):
        p = None if pred is None else s[0:1].fill_(pred)
        fq = F.FusedQuant(q8, s[0:1], ws, E4, bias_pred=p, amax_bits=s[1:2], flags=s[2:3])
        o = blank(c.rows, heads * dh, gpu)
        F.llama_cache_attention(qd, cache, seqs, heads, c.max_rows, window=window, o=o, fq=fq)
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), outs[0].view(torch.int16)) and torch.equal(q8[:live], rq)
        assert s.cpu().tolist() == [int(rb.item()), int(ra.item()), int(rf.item())]
        assert (q8[live:] == 0x55).all() and counts(ws) == 0


def test_shares_keep_nan_where_it_is_seen(gpu):
    """NaN and infinities behind one sequence's rows, among the values of another."""
    say("shares, nan")
    c = Case(52, 4, 2, 128, E4, 1024, [1, 1, 2], [3000, 700, 900], capacity=350)
    q = rand_bits(c.rng, (c.rows, 512))
    cache, seqs = c.device(gpu)
    clean = np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 2))
    page, slot = C.place(c.host, c.pages, 2, 899)     # the second row of sequence 2 only
    cache.v[page, 1, slot // 16, 5, slot % 16] = 0x7F
    got = np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 2))
    page, slot = C.place(c.host, c.pages, 1, 300)     # every row of sequence 1
    cache.k[page, 0, slot, 9] = 0x7F
    both = np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 2))
    torch.cuda.synchronize()
    nan = np.zeros(clean.shape, dtype=bool)
    nan[3, [2 * 128 + 5, 3 * 128 + 5]] = True         # heads of key/value head 1
    assert ((got & 0x7FFF) > 0x7F80)[nan].all() and np.array_equal(got[~nan], clean[~nan])
    nan[1, :256] = True
    assert ((both & 0x7FFF) > 0x7F80)[nan].all() and np.array_equal(both[~nan], clean[~nan])


#   heads kv dh fmt page capacity new total window
PARTS = [
    (8, 1, 128, E4, 64, 500, [1], [20001], 0),                 # 469 tiles in 30 parts
    (4, 4, 128, E5, 16, None, [1], [3000], 0),
    (8, 8, 64, BF, 64, None, [1, 1, 1], [2000, 40, 0], 0),     # parts that have nothing
    (2, 2, 128, E4, 1024, 60, [1], [33], 0),                   # a short one under a long table
    (2, 2, 128, E4, 64, 200, [1, 1], [7000, 300], 1000),       # a window of a few tiles
    (2, 2, 128, E4, 64, 200, [1], [0], 0),
    (2, 2, 64, E4, 64, 200, [4], [4000], 0),
    (10, 10, 64, E4, 32, None, [1] * 25, [30 * i for i in range(25)], 0),     # 250 items
    (9, 9, 64, E4, 32, None, [1] * 33, [11 * i for i in range(33)], 0),       # 297: the longest first
    (8, 8, 64, E5, 32, None, [1] * 64, [(37 * i) % 500 for i in range(64)], 0),  # 512
    (8, 8, 64, E5, 32, None, [1] * 65, [(37 * i) % 500 for i in range(65)], 0),
]


@pytest.mark.parametrize("heads,kv,dh,fmt,page,capacity,new,total,window", PARTS)
def test_parts(gpu, heads, kv, dh, fmt, page, capacity, new, total, window):
    say("parts", heads, kv, dh, fmt, page, capacity, new[:4], total[:4], window)
    c = Case(53, heads, kv, dh, fmt, page, new, total, 1, capacity=capacity)
    c.poison_unused()
    q = rand_bits(c.rng, (c.rows, heads * dh))
    cache, seqs = c.device(gpu)
    ws = F.cache_attention_workspace(c.rows, heads, cache, seqs, c.max_rows)
    for _ in range(2):
        o = blank(c.rows, heads * dh, gpu)
        F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, heads, c.max_rows, window=window, o=o, ws=ws)
        torch.cuda.synchronize()
        check(c, q, o, window)
        assert counts(ws) == 0


@pytest.mark.parametrize("window", [0, 1, 63, 600, 2 ** 30 - 1, 2 ** 30, 2 ** 63 - 1])
def test_chunk_ranges_and_windows(gpu, window):
    """A chunk whose keys are cut into ranges; windows up to the largest number."""
    say("chunk ranges", window)
    c = Case(54, 4, 2, 128, E4, 64, [150, 70], [4100, 1500], 2)
    c.poison_unused()
    q = rand_bits(c.rng, (c.rows, 512))
    cache, seqs = c.device(gpu)
    o = blank(c.rows, 512, gpu)
    ws = F.cache_attention_workspace(c.rows, 4, cache, seqs, 150)
    F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 150, window=window, o=o, ws=ws)
    torch.cuda.synchronize()
    check(c, q, o, window if window < 2 ** 30 else 0)
    assert counts(ws) == 0


def test_largest_max_rows(gpu):
    say("largest max_rows")
    c = Case(55, 4, 2, 128, E4, 64, [1, 40], [100, 300])
    q = rand_bits(c.rng, (c.rows, 512))
    cache, seqs = c.device(gpu)
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 2 ** 62)
    torch.cuda.synchronize()
    check(c, q, o)


def test_one_workspace_for_calls_of_all_sizes(gpu):
    """One after the other on a stream, twice around: each as with its own."""
    say("one workspace")
    cases = [Case(56, 16, 8, 128, E4, 1024, [1] * 6, [1, 3000, 64, 0, 777, 900], capacity=48),
             Case(57, 8, 1, 128, E5, 64, [1], [9001], capacity=500),
             Case(58, 4, 2, 64, BF, 64, [150, 1], [1900, 700]),
             Case(59, 16, 4, 128, E4, 512, [1] * 30 + [50], lens(6, 30, 700) + [400], capacity=40)]
    devs = [c.device(gpu) for c in cases]
    qs = [strided(rand_bits(c.rng, (c.rows, c.heads * c.d_head)), gpu, 0) for c in cases]
    sizes = [F.llama_cache_attention_ws_bytes(c.rows, c.heads, *d, c.max_rows) for c, d in zip(cases, devs)]
    ws = torch.zeros((max(sizes),), dtype=torch.uint8, device=gpu)
    want = [F.llama_cache_attention(q, *d, c.heads, c.max_rows) for q, d, c in zip(qs, devs, cases)]
    for _ in range(2):
        for q, d, c, w in zip(qs, devs, cases, want):
            o = F.llama_cache_attention(q, *d, c.heads, c.max_rows, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(o, w) and counts(ws) == 0


def test_graphs_that_share_a_workspace(gpu):
    """Two captured calls, of shares and of parts, replayed in turn on one stream,
    with eager work among them."""
    say("graphs sharing a workspace")
    cases = [Case(60, 16, 8, 128, E4, 1024, [1] * 6, [1, 3000, 64, 0, 777, 900], capacity=48),
             Case(61, 8, 1, 128, E5, 64, [1], [9001], capacity=500)]
    devs = [c.device(gpu) for c in cases]
    qs = [strided(rand_bits(c.rng, (c.rows, c.heads * c.d_head)), gpu, 0) for c in cases]
    sizes = [F.llama_cache_attention_ws_bytes(c.rows, c.heads, *d, c.max_rows) for c, d in zip(cases, devs)]
    ws = torch.zeros((max(sizes),), dtype=torch.uint8, device=gpu)
    outs = [torch.zeros_like(q) for q in qs]
    graphs = []
    for q, d, c, o in zip(qs, devs, cases, outs):
        F.llama_cache_attention(q, *d, c.heads, c.max_rows, o=o, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            F.llama_cache_attention(q, *d, c.heads, c.max_rows, o=o, ws=ws)
        graphs.append(g)
    for t in range(4):
        for o in outs:
            o.zero_()
        for d, c in zip(devs, cases):       # other lengths, from which the work is cut anew
            d[1].kv_len.copy_(torch.from_numpy(np.maximum(c.kv_len - 130 * t, 0)).to(gpu))
        for g in graphs + graphs:
            g.replay()
        want = [F.llama_cache_attention(q, *d, c.heads, c.max_rows) for q, d, c in zip(qs, devs, cases)]
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want)) and counts(ws) == 0


def test_inconsistent_rows_stay_inside(gpu):
    """cu_rows that falls, starts behind 0 or runs beyond the rows: what is written is
    inside the call's rows and the pages of the tables."""
    say("inconsistent rows")
    for cu in ([0, 40, 10, 60], [7, 9, 9, 20], [0, 2 ** 31 - 1, 5, 2 ** 31 - 1], [-2 ** 31, -5, 3, 50], [60, 40, 20, 0]):
        c = Case(62, 4, 2, 128, E4, 16, [20, 20, 20], [70, 200, 33], spare=5)
        cache, seqs = c.device(gpu)
        seqs.cu_rows.copy_(torch.tensor(cu, dtype=torch.int32))
        before = {n: getattr(cache, n).clone() for n in ("k", "v", "k_exp", "v_exp")}
        wide = torch.full((70, 512), SENTINEL, dtype=torch.int16, device=gpu).view(torch.bfloat16)
        x = strided(rand_bits(c.rng, (60, 8 * 128)), gpu, 0)
        q = F.llama_cache_append(x, cache, seqs, 4, table=c.table(gpu))
        F.llama_cache_attention(q, cache, seqs, 4, 60, o=wide[5:65])
        k = torch.full((70, 256), SENTINEL, dtype=torch.int16, device=gpu).view(torch.bfloat16)
        F.llama_cache_read(cache, seqs, 60, k=k[5:65])
        torch.cuda.synchronize()
        for t in (wide, k):
            assert (np_bits(t)[:5] == SENTINEL).all() and (np_bits(t)[65:] == SENTINEL).all()
        used = set(c.pages[(c.pages >= 0) & (c.pages < cache.n_pages)].tolist())
        free = [p for p in range(cache.n_pages) if p not in used]
        assert len(free) == 5
        for n, t in before.items():
            assert torch.equal(getattr(cache, n)[free], t[free]), n


def test_first_sequence_behind_row_0(gpu):
    """Rows before cu_rows[0] belong to no sequence: they are left, those behind are right."""
    say("rows before the first sequence")
    c = Case(64, 4, 2, 128, E4, 64, [700, 130, 1], [700, 300, 65])
    q = rand_bits(c.rng, (c.rows, 512))
    cache, seqs = c.device(gpu)
    seqs = F.CacheSeqs(seqs.cu_rows[1:], seqs.kv_len[1:], seqs.pages[1:])
    o = blank(c.rows, 512, gpu)
    F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 700, o=o)
    k, v = blank(c.rows, 256, gpu), blank(c.rows, 256, gpu)
    F.llama_cache_read(cache, seqs, c.rows, k=k, v=v)
    torch.cuda.synchronize()
    for t in (o, k, v):
        assert (np_bits(t)[:700] == SENTINEL).all()
    want, mean, top = C.attention(q, c.host, c.cu[1:], c.kv_len[1:], c.pages[1:], 4)
    err = np.abs(D.bf16_to_f64(np_bits(o)) - want)
    assert (err <= bound(c, want, mean, top))[700:].all()
    wk, wv = C.read(c.host, c.cu[1:], c.kv_len[1:], c.pages[1:], c.rows)
    assert np.array_equal(np_bits(k)[700:], wk[700:]) and np.array_equal(np_bits(v)[700:], wv[700:])


def test_another_stream_needs_a_workspace(gpu):
    say("another stream")
    c = Case(66, 8, 2, 128, E4, 16, [1, 30], [900, 200])
    cache, seqs = c.device(gpu)
    q = strided(rand_bits(c.rng, (c.rows, 1024)), gpu, 0)
    want = F.llama_cache_attention(q, cache, seqs, 8, 30)
    ws, o = F.cache_attention_workspace(c.rows, 8, cache, seqs, 30), torch.zeros_like(q)
    st = torch.cuda.Stream()
    with pytest.raises(ValueError):
        F.llama_cache_attention(q, cache, seqs, 8, 30, o=o, stream=st)
    torch.cuda.synchronize()
    F.llama_cache_attention(q, cache, seqs, 8, 30, o=o, ws=ws, stream=st)
    st.synchronize()
    assert torch.equal(o, want)
    with torch.cuda.stream(st):
        o2 = F.llama_cache_attention(q, cache, seqs, 8, 30)
    st.synchronize()
    assert torch.equal(o2, want)


def test_append_without_queries(gpu):
    """The C call with q NULL writes the same cache."""
    say("append without queries")
    for fmt, new, total in ((E4, [1, 30], [9, 77]), (BF, [130], [130])):
        c = Case(63, 8, 2, 128, fmt, 32, new, total)
        (a, sa), (b, sb) = c.device(gpu), c.device(gpu)
        x = strided(rand_bits(c.rng, (c.rows, 12 * 128)), gpu, 8)
        table = c.table(gpu)
        F.llama_cache_append(x, a, sa, 8, table=table)
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        st = F.lib().llama_cache_append(ctypes.c_void_p(x.data_ptr()), c.rows, x.stride(0), 8, ctypes.byref(b._c),
                                        ctypes.byref(sb._c), ctypes.c_void_p(table.data_ptr()),
                                        c.max_pages * 32, None, 0, stream)
        assert st == 0
        torch.cuda.synchronize()
        for n in ("k", "v", "k_exp", "v_exp"):
            t = getattr(a, n)
            assert t is None or torch.equal(t.view(torch.uint8), getattr(b, n).view(torch.uint8)), n


@pytest.mark.parametrize("fmt,new,total", [(E4, [1, 1], [900, 70]), (BF, [1], [3000]), (E4, [90], [400]),
                                           (BF, [130, 1], [500, 300]), (E4, [200], [2000])])
def test_scores_beyond_what_their_exponents_hold(gpu, fmt, new, total):
    """Scores of 2^40 to 2^43, exact in fp32: the largest one takes all, ties share."""
    say("large scores", fmt, new, total)
    c = Case(65, 4, 2, 128, fmt, 64, new, total)
    h = c.host
    if fmt == BF:
        h.k[...] = 0
        h.k[..., 0] = C.round_bf16(c.rng.integers(1, 8, h.k[..., 0].shape).astype(np.float64))
    else:
        h.k[...] = 0
        h.k[..., 0] = c.rng.integers(0x38, 0x50, h.k[..., 0].shape)      # 1 to 7.5
        h.k_exp[...] = 127
    q = np.zeros((c.rows, 512), dtype=np.uint16)
    q[:, ::128] = C.round_bf16(np.full((c.rows, 4), 2.0 ** 40))
    cache, seqs = c.device(gpu)
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, c.max_rows)
    torch.cuda.synchronize()
    want, mean, _ = C.attention(q, h, c.cu, c.kv_len, c.pages, 4)
    # the weights are 1 and 0: sums of the winners in fp32, one rounding; two for P = 1 (exact)
    lim = 2.0 ** -8 * np.abs(want) + (2.0 ** -7 + max(total) * 2.0 ** -23) * mean
    assert (np.abs(D.bf16_to_f64(np_bits(o)) - want) <= lim).all()


@pytest.mark.parametrize("fmt", [E4, BF])
def test_cache_beyond_32_bit_offsets(gpu, fmt):
    """Pages at the ends of a cache of 5.2 (bf16: 10.5) GB for keys and for values: the
    bits of a small cache."""
    say("large cache", fmt)
    n_pages, kv, page = 80000, 8, 64
    big, small = F.KVCache(n_pages, kv, 128, page, fmt, gpu), F.KVCache(8, kv, 128, page, fmt, gpu)
    far = torch.tensor([[n_pages - 1, 0, 65536, -1], [32768, n_pages - 2, 40001, 1]], dtype=torch.int32, device=gpu)
    near = torch.tensor([[0, 1, 2, -1], [3, 4, 5, 6]], dtype=torch.int32, device=gpu)
    table = F.llama_rope_table(4 * page, 128, device=gpu)
    outs = []
    for cache, pages in ((big, far), (small, near)):
        rng = np.random.default_rng(67)
        got = []
        for new, total in (([150, 200], [150, 200]), ([1, 1], [151, 201]), ([1, 40], [152, 241])):
            cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=gpu)
            seqs = F.CacheSeqs(cu, torch.tensor(total, dtype=torch.int32, device=gpu), pages)
            x = strided(rand_bits(rng, (sum(new), 24 * 128)), gpu, 0)
            q = F.llama_cache_append(x, cache, seqs, 8, table=table)
            got += [q, F.llama_cache_attention(q, cache, seqs, 8, max(new)), *F.llama_cache_read(cache, seqs, sum(new))]
        outs.append(got)
    torch.cuda.synchronize()
    for a, b in zip(*outs):
        assert torch.isfinite(a.float()).all() and torch.equal(a, b)
