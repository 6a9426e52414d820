"""GPU parity of the paged key/value cache calls with oracle/cache.py.

Bars, from the arithmetic:
  * append: bit for bit.  The rotation is done in fp64 (its products are exact
    there), rounded to fp32; bias, codes and exponents are integer work, and
    the bf16 roundings of the queries, keys and values are from that fp32 value.
  * read: bit for bit (codes times a power of two).
  * attention, per element, with A the softmax-weighted mean of |v| and T the
    largest sum_d |q_d k_d| / sqrt(d) of the row's keys:
      scores: an fp32 sum of d products is off by at most d 2^-24 T; the scaled
      score is rounded once more, and so is its difference to the maximum
      (4 2^-24 T together).  ds = (d + 4) 2^-24 T is the error of a score; a
      probability is off by the factor exp(2 ds) at most, as is their sum: 4 ds A
      in the result (first order; 8 ds A for the rest);
      probabilities: rounded to bf16, 2^-8 A; their fp32 sums over n keys:
      n 2^-24 A each, and exp2's own error (2^-22) twice;
      the result rounded to bf16: 2^-8 of its value.
"""
import numpy as np
import pytest
import torch

from cache_cases import SENTINEL, Case, blank, rand_bits, strided
from oracle import cache as C
from oracle import decoder as D
from paper_2309_17224_amd import fp8lin as F
from parity_util import np_bits

pytestmark = pytest.mark.gpu

E4, E5, BF = F.E4M3, F.E5M2, F.CACHE_BF16


def say(*a):
    print("\n[case]", *a, flush=True)


def host_arrays(cache):
    return {n: (np_bits(t) if t is not None else None) for n, t in
            (("k", cache.k), ("v", cache.v), ("k_exp", cache.k_exp), ("v_exp", cache.v_exp))}


# ------------------------------------------------------------------ append and read
#   heads kv dh  fmt page new            total            tail
APPEND = [
    (4, 2, 128, E4, 16, [1], [1], 0),
    (4, 2, 128, E4, 16, [1], [33], 2),
    (8, 2, 128, E5, 32, [1, 1, 1], [1, 16, 17], 0),
    (3, 1, 128, E4, 16, [16], [16], 0),
    (4, 4, 128, E5, 64, [37], [50], 5),
    (4, 2, 128, BF, 16, [17, 1, 40], [20, 31, 40], 1),
    (12, 12, 64, E4, 16, [5, 33], [7, 64], 0),
    (6, 3, 64, E5, 128, [100], [261], 3),
    (2, 1, 64, BF, 16, [1, 15, 16, 17], [1, 15, 32, 49], 0),
    (5, 5, 64, BF, 1024, [70], [1100], 0),
    (8, 2, 128, E4, 16, [0, 3, 0, 0, 2, 0], [0, 3, 12, 0, 2, 5], 1),
    (4, 2, 128, E4, 16, [1] * 70, list(range(1, 71)), 0),          # more sequences than lanes of a wave
    (4, 1, 64, E4, 32, [2] * 65 + [131], [9] * 65 + [150], 0),
    (4, 2, 128, E5, 16, [6, 4], [3, 2], 0),                        # positions below 0
]


@pytest.mark.parametrize("heads,kv,dh,fmt,page,new,total,tail", APPEND)
@pytest.mark.parametrize("rot", [True, False])
def test_append_and_read(gpu, heads, kv, dh, fmt, page, new, total, tail, rot):
    say("append", heads, kv, dh, fmt, page, new[:4], total[:4], tail, rot)
    c = Case(7, heads, kv, dh, fmt, page, new, total, tail)
    x = rand_bits(c.rng, (c.rows, (heads + 2 * kv) * dh), 2.0)
    cache, seqs = c.device(gpu)
    qkv = strided(x, gpu, 24)
    table = c.table(gpu) if rot else None
    q = blank(c.rows, heads * dh, gpu, 16)
    assert F.llama_cache_append(qkv, cache, seqs, heads, table=table, q=q) is q
    k, v = blank(c.rows, kv * dh, gpu, 8), blank(c.rows, kv * dh, gpu)
    F.llama_cache_read(cache, seqs, c.rows, k=k, v=v)
    torch.cuda.synchronize()
    tab = table.cpu().numpy().reshape(-1, dh // 2, 2) if rot else None
    want = C.append(x, c.host, c.cu, c.kv_len, c.pages, heads, tab)
    live = int(c.cu[-1])
    assert np.array_equal(np_bits(q)[:live], want[:live])
    for name, got in host_arrays(cache).items():
        ref = getattr(c.host, name)
        assert (got is None) == (ref is None)
        assert got is None or np.array_equal(got, ref), name
    wk, wv = C.read(c.host, c.cu, c.kv_len, c.pages, c.rows)
    assert np.array_equal(np_bits(k)[:live], wk[:live]) and np.array_equal(np_bits(v)[:live], wv[:live])
    for t in (q, k, v):   # rows behind the last sequence, and what lies between rows, are left
        assert (np_bits(t)[live:] == SENTINEL).all()
        if t._base is not None:
            assert (t._base.view(torch.int16)[:, t.shape[1]:] == SENTINEL).all()
    assert np.array_equal(np_bits(qkv), x)


def test_append_in_place_and_absent_pages(gpu):
    say("append in place")
    c = Case(8, 4, 2, 128, E4, 16, [40, 3], [45, 18], capacity=3)
    c.pages[0, 1] = c.host.n_pages        # positions 16 .. 31 of sequence 0 absent
    c.pages[1, 1] = -5
    x = rand_bits(c.rng, (c.rows, 8 * 128))
    cache, seqs = c.device(gpu)
    qkv = strided(x, gpu, 0)
    F.llama_cache_append(qkv, cache, seqs, 4, table=c.table(gpu), q=qkv[:, :512])
    k, v = F.llama_cache_read(cache, seqs, c.rows)
    torch.cuda.synchronize()
    want = C.append(x, c.host, c.cu, c.kv_len, c.pages, 4, c.table(gpu).cpu().numpy().reshape(-1, 64, 2))
    got = np_bits(qkv)
    assert np.array_equal(got[:, :512], want) and np.array_equal(got[:, 512:], x[:, 512:])
    assert not want[11:27].any()
    for name, a in host_arrays(cache).items():
        assert np.array_equal(a, getattr(c.host, name)), name
    wk, wv = C.read(c.host, c.cu, c.kv_len, c.pages, c.rows)
    assert np.array_equal(np_bits(k), wk) and np.array_equal(np_bits(v), wv)


@pytest.mark.parametrize("fmt", [E4, E5, BF])
def test_append_special_values(gpu, fmt):
    """Zero rows, one huge or tiny value, infinities and NaN: codes and exponents
    are the oracle's (bias 0 for a zero, infinite or NaN amax; b <= 126)."""
    say("append special", fmt)
    c = Case(9, 2, 2, 64, fmt, 16, [12], [12])
    x = rand_bits(c.rng, (12, 6 * 64))
    kv = x[:, 2 * 64:]
    kv[1] = 0
    kv[2, 5::64] = 0x7F7F          # largest finite
    kv[3] = 0x0001                 # smallest subnormal
    kv[4, 3::64] = 0x7F80          # +inf
    kv[5, 3::64] = 0xFF80
    kv[6, 7::64] = 0x7FC1          # NaN
    kv[7, 7::64] = 0xFFC1
    kv[8] = 0x8000
    kv[9] &= 0x80FF                # tiny
    cache, seqs = c.device(gpu)
    F.llama_cache_append(strided(x, gpu, 0), cache, seqs, 2)
    torch.cuda.synchronize()
    C.append(x, c.host, c.cu, c.kv_len, c.pages, 2, None)
    got = host_arrays(cache)
    if fmt == BF:
        # values are copied; keys go through fp32, which keeps NaN a NaN
        assert np.array_equal(got["v"], c.host.v)
        a, b = D.bf16_to_f64(got["k"]), D.bf16_to_f64(c.host.k)
        assert np.array_equal(a, b, equal_nan=True)
        return
    for name in ("k_exp", "v_exp", "k", "v"):
        assert np.array_equal(got[name], getattr(c.host, name)), name


def test_append_overwrites_only_its_slots(gpu):
    """Token by token through two blocks: earlier tokens of a block keep theirs."""
    say("append token by token")
    c = Case(10, 2, 1, 128, E4, 16, [1], [21])
    cache, seqs = c.device(gpu)
    table = c.table(gpu)
    tab = table.cpu().numpy().reshape(-1, 64, 2)
    for n in range(1, 22):
        x = rand_bits(c.rng, (1, 4 * 128))
        seqs.kv_len.fill_(n)
        F.llama_cache_append(strided(x, gpu, 0), cache, seqs, 2, table=table)
        C.append(x, c.host, c.cu, [n], c.pages, 2, tab)
    torch.cuda.synchronize()
    for name, a in host_arrays(cache).items():
        assert np.array_equal(a, getattr(c.host, name)), name


def test_read_one_output(gpu):
    say("read one output")
    c = Case(11, 4, 4, 64, E4, 32, [50], [90])
    cache, seqs = c.device(gpu)
    wk, wv = C.read(c.host, c.cu, c.kv_len, c.pages, c.rows)
    k, none = F.llama_cache_read(cache, seqs, c.rows, want_v=False)
    assert none is None and np.array_equal(np_bits(k), wk)
    none, v = F.llama_cache_read(cache, seqs, c.rows, want_k=False)
    assert none is None and np.array_equal(np_bits(v), wv)


# ------------------------------------------------------------------ attention
def bound(c, want, mean, top):
    """Largest allowed difference of each element (see the module's docstring)."""
    n, d = max(int(c.kv_len.max()), 1), c.d_head
    ds = np.repeat((d + 4) * 2.0 ** -24 * top, d, axis=1)
    off = (8 * ds + 2.0 ** -8 + 2 * n * 2.0 ** -24 + 2.0 ** -20) * mean
    return off + 2.0 ** -8 * (np.abs(want) + off) + 1e-30


def check(c, q, o, window=0, max_rows=None, what=""):
    want, mean, top = C.attention(q, c.host, c.cu, c.kv_len, c.pages, c.heads, max_rows, window)
    got = D.bf16_to_f64(np_bits(o))
    live = np.zeros(c.rows, dtype=bool)
    for s in range(len(c.kv_len)):
        n = int(c.cu[s + 1] - c.cu[s])
        live[c.cu[s]:c.cu[s] + (n if max_rows is None else min(n, max_rows))] = True
    assert (np_bits(o)[~live] == SENTINEL).all()
    err, lim = np.abs(got - want)[live], bound(c, want, mean, top)[live]
    worst = float((err / lim).max()) if err.size else 0.0
    den = np.linalg.norm(want[live])
    print(f"{what} worst {worst:.3f} of the bound, rel {np.linalg.norm((got - want)[live]) / max(den, 1e-30):.2e}", flush=True)
    assert np.isfinite(got[live]).all() and worst <= 1.0
    return want


#   heads kv dh  fmt page new total tail window
ATTEND = [
    (4, 2, 128, E4, 16, [1], [1], 0, 0),
    (4, 2, 128, E4, 16, [1], [2], 1, 0),
    (8, 2, 128, E4, 16, [1], [300], 0, 0),
    (8, 1, 128, E5, 32, [1, 1, 1], [63, 64, 65], 2, 0),
    (64, 8, 128, E4, 64, [1], [1500], 0, 0),
    (4, 4, 128, E4, 16, [1, 1], [17, 1000], 0, 0),                 # no groups
    (16, 1, 128, E5, 128, [1], [777], 0, 0),
    (40, 2, 128, E4, 16, [1, 1], [129, 513], 0, 0),                # 20 heads on one
    (28, 4, 128, E4, 16, [1, 2], [140, 90], 0, 0),                 # groups of 7
    (12, 12, 64, E4, 16, [1, 1, 1], [1, 200, 431], 0, 0),
    (8, 2, 64, BF, 32, [1, 1], [100, 257], 0, 0),
    (8, 2, 128, BF, 16, [1], [600], 0, 0),
    (4, 2, 128, E4, 16, [3], [3], 0, 0),
    (4, 2, 128, E4, 16, [16], [16], 0, 0),
    (8, 2, 128, E4, 16, [64], [64], 0, 0),
    (8, 2, 128, E5, 64, [65], [190], 3, 0),
    (8, 2, 128, BF, 16, [130], [131], 0, 0),
    (4, 4, 128, E4, 16, [150, 129], [150, 300], 0, 0),
    (6, 2, 64, E4, 16, [100], [333], 0, 0),                        # groups of 3
    (12, 12, 64, BF, 64, [77, 1, 140], [77, 400, 222], 5, 0),
    (2, 1, 64, E5, 1024, [257], [600], 0, 0),
    (8, 2, 128, E4, 16, [40, 1, 0, 9, 1], [40, 333, 0, 200, 1], 1, 0),
    (4, 2, 128, E4, 32, [90], [400], 0, 100),                      # windows
    (4, 2, 128, BF, 16, [1, 1], [400, 30], 0, 64),
    (4, 2, 64, E5, 16, [33], [200], 0, 1),
    (8, 8, 128, E4, 16, [70], [500], 0, 65),
    (4, 2, 128, E4, 16, [6, 4, 20], [3, 0, 12], 0, 0),             # positions below 0: empty rows
    (4, 1, 128, E4, 16, [1] * 70, [3 * i + 1 for i in range(70)], 0, 0),
    (16, 2, 128, E4, 16, [2, 2], [600, 65], 0, 0),                 # two tokens, 16 rows a head
    (8, 1, 128, E4, 16, [4], [500], 0, 0),                         # 32 rows a head
    (128, 1, 64, E4, 16, [1], [200], 0, 0),
]


@pytest.mark.parametrize("heads,kv,dh,fmt,page,new,total,tail,window", ATTEND)
def test_attention(gpu, heads, kv, dh, fmt, page, new, total, tail, window):
    say("attention", heads, kv, dh, fmt, page, new[:4], total[:4], tail, window)
    c = Case(21, heads, kv, dh, fmt, page, new, total, tail)
    c.poison_unused()              # what no sequence holds is NaN
    q = rand_bits(c.rng, (c.rows, heads * dh))
    cache, seqs = c.device(gpu)
    o = blank(c.rows, heads * dh, gpu, 8)
    F.llama_cache_attention(strided(q, gpu, 16), cache, seqs, heads, c.max_rows, window=window, o=o)
    first = np_bits(o).copy()
    check(c, q, o, window)
    # max_rows is a bound: a larger one gives the same rows; the same call the same bits
    o2, o3 = blank(c.rows, heads * dh, gpu), blank(c.rows, heads * dh, gpu)
    qd = strided(q, gpu, 0)
    F.llama_cache_attention(qd, cache, seqs, heads, c.max_rows + 37, window=window, o=o2)
    F.llama_cache_attention(qd, cache, seqs, heads, c.max_rows, window=window, o=o3)
    torch.cuda.synchronize()
    check(c, q, o2, window, what="larger max_rows:")
    assert np.array_equal(np_bits(o3), first)


@pytest.mark.parametrize("heads,kv,dh,fmt,page,new,total", [
    (64, 8, 128, E4, 64, [1, 1], [4097, 1200]),
    (8, 8, 128, E5, 16, [1], [5000]),
    (8, 1, 128, BF, 64, [5], [3001]),
    (8, 2, 128, E4, 32, [300], [2500]),
    (4, 4, 64, BF, 16, [500], [1800]),
])
def test_attention_long(gpu, heads, kv, dh, fmt, page, new, total):
    say("attention long", heads, kv, dh, fmt, page, new, total)
    c = Case(22, heads, kv, dh, fmt, page, new, total)
    q = rand_bits(c.rng, (c.rows, heads * dh))
    cache, seqs = c.device(gpu)
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, heads, c.max_rows)
    check(c, q, o)


def test_attention_sharp_and_flat_scores(gpu):
    """Scores of hundreds, where one key takes all, and of zero, where all are equal."""
    say("attention sharp")
    c = Case(23, 4, 2, 128, E4, 16, [20, 1], [300, 300])
    q = rand_bits(c.rng, (c.rows, 512), 40.0)
    q[3] = 0
    q[20, :128] = 0
    cache, seqs = c.device(gpu)
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, 20)
    check(c, q, o)


def test_attention_values_of_very_different_scales(gpu):
    """Tokens whose values are 2^-40 and 2^30 of the others', rows of large and tiny queries."""
    say("attention scales")
    c = Case(24, 8, 2, 128, E4, 16, [1, 33], [200, 100])
    c.host.v_exp[:, :, 3] -= 40
    c.host.v_exp[:, :, 7] += 30
    c.host.k_exp[:, :, 5] -= 20
    q = rand_bits(c.rng, (c.rows, 1024))
    q[2] = rand_bits(c.rng, (1024,), 1e-30)
    q[5] = rand_bits(c.rng, (1024,), 30.0)
    q[6, ::7] = 0x0001             # subnormals beside ordinary values
    cache, seqs = c.device(gpu)
    o = F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 8, 33)
    check(c, q, o)


def test_attention_absent_pages(gpu):
    """Pages taken out of the table, at the start, in the middle, at the end and all
    of a sequence: their tokens are not seen, and rows that see none give 0."""
    say("attention absent pages")
    for new in ([1, 1, 1, 1], [40, 17, 70, 5]):
        c = Case(25, 8, 2, 128, E4, 16, new, [200, 100, 150, 60])
        c.pages[0, 0:3] = [-1, c.host.n_pages, 2 ** 31 - 1]
        c.pages[0, 7] = -2 ** 31
        c.pages[1, 6] = -1
        c.pages[2, ::2] = -7
        c.pages[3] = -1
        c.poison_unused()
        q = rand_bits(c.rng, (c.rows, 1024))
        cache, seqs = c.device(gpu)
        o = blank(c.rows, 1024, gpu)
        F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 8, max(new), o=o)
        want = check(c, q, o)
        assert not want[c.cu[3]:].any() and not np_bits(o)[c.cu[3]:].any()


def test_attention_longer_than_its_table(gpu):
    """kv_len beyond what the page table holds: the keys that it holds are seen."""
    say("attention beyond the table")
    for new in ([1, 1], [30, 50]):
        c = Case(26, 4, 2, 128, E5, 16, new, [90, 64], capacity=4)
        q = rand_bits(c.rng, (c.rows, 512))
        cache, seqs = c.device(gpu)
        o = blank(c.rows, 512, gpu)
        F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, max(new), o=o)
        check(c, q, o)
    seqs.kv_len.copy_(torch.tensor([2 ** 31 - 1, -2 ** 31], dtype=torch.int32))
    F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, max(new), o=o)
    torch.cuda.synchronize()
    assert not np_bits(o)[c.cu[1]:].any()


@pytest.mark.parametrize("fmt", [E4, BF])
def test_attention_nan_stays_where_it_is_seen(gpu, fmt):
    """A NaN (bf16: infinities too) in a later token's key or value reaches only
    the rows that see the token, in the value only its own column."""
    say("attention nan", fmt)
    for new, total, at in (([40], [150], 140), ([5], [100], 97), ([70], [70], 33)):
        for where in ("v", "k"):
            c = Case(27, 4, 2, 128, fmt, 16, new, total)
            q = rand_bits(c.rng, (c.rows, 512))
            cache, seqs = c.device(gpu)
            clean = np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, new[0])).copy()
            g, slot = C.place(c.host, c.pages, 0, at)
            nan = 0x7FC0 if fmt == BF else 0x7F
            bits = torch.int16 if fmt == BF else torch.uint8
            if where == "v":
                cache.v.view(bits)[g, 1, slot // 16, 9, slot % 16] = nan
                if fmt == BF:
                    cache.v.view(bits)[g, 0, slot // 16, 5, slot % 16] = 0x7F80
                    cache.v.view(bits)[g, 0, slot // 16, 6, slot % 16] = -128     # 0xFF80
            else:
                cache.k.view(bits)[g, 1, slot, 9] = nan
            got = np_bits(F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 4, new[0]))
            first = at - (total[0] - new[0])      # the first row that sees it
            assert np.array_equal(got[:first], clean[:first])
            f = D.bf16_to_f64(got).reshape(-1, 4, 128)
            if where == "v":
                assert np.isnan(f[first:, 2:, 9]).all()
                f[:, 2:, 9] = 0
                if fmt == BF:
                    assert (f[first:, :2, 5] == np.inf).all() and (f[first:, :2, 6] == -np.inf).all()
                    f[:, :2, 5:7] = 0
                assert np.isfinite(f).all()
            else:
                assert np.isnan(f[first:, 2:]).all() and np.isfinite(f[:, :2]).all()


def test_attention_max_rows_bounds_the_rows(gpu):
    """Rows after the first max_rows of a sequence are left as they were."""
    say("attention max_rows")
    for m in (1, 3, 20):
        c = Case(28, 8, 2, 128, E4, 16, [30, 2], [50, 40])
        q = rand_bits(c.rng, (c.rows, 1024))
        cache, seqs = c.device(gpu)
        o = blank(c.rows, 1024, gpu)
        F.llama_cache_attention(strided(q, gpu, 0), cache, seqs, 8, m, o=o)
        check(c, q, o, max_rows=m)


# ------------------------------------------------------------------ fused quantise
@pytest.mark.parametrize("new,total", [([1], [700]), ([1, 1, 1], [64, 1, 900]), ([200], [300]), ([33, 1], [33, 2000])])
@pytest.mark.parametrize("fmt", [F.E4M3, F.E5M2, F.E4_A])
def test_attention_quantise(gpu, new, total, fmt):
    """Codes, bias, amax and flags are those of fp8_quantise of the output's live
    rows, whatever the prediction; rows behind them are left."""
    say("attention quantise", new, total, fmt)
    c = Case(31, 8, 2, 128, E4, 64, new, total, tail=2)
    cols, live = 1024, int(c.cu[-1])
    q = strided(rand_bits(c.rng, (c.rows, cols)), gpu, 0)
    cache, seqs = c.device(gpu)
    ref = F.llama_cache_attention(q, cache, seqs, 8, c.max_rows)
    rq, _, rb, ra, rf = F.fp8_quantise(ref[:live], fmt, 1)
    exact = int(rb.item())
    for pred in (None, exact, exact + 3, exact - 2):
        q8 = torch.full((c.rows, cols + 8), 0x55, dtype=torch.uint8, device=gpu)[:, :cols]
        s = torch.zeros(3, dtype=torch.int32, device=gpu)
        p = None if pred is None else s[0:1].fill_(pred)
        ws = F.cache_attention_workspace(c.rows, 8, cache, seqs, c.max_rows)
        fq = F.FusedQuant(q8, s[0:1], ws, fmt, 1, bias_pred=p, amax_bits=s[1:2], flags=s[2:3])
        o = blank(c.rows, cols, gpu)
        F.llama_cache_attention(q, cache, seqs, 8, c.max_rows, o=o, fq=fq)
        torch.cuda.synchronize()
        assert torch.equal(o[:live], ref[:live]) and (np_bits(o)[live:] == SENTINEL).all()
        assert s.cpu().tolist() == [exact, int(ra.item()), int(rf.item())]
        assert torch.equal(q8[:live], rq)
        assert (q8[live:] == 0x55).all()


def test_attention_quantise_of_nothing(gpu):
    """Every row empty, or no sequence at all: amax 0, bias 0 and the zero flag."""
    say("attention quantise of nothing")
    c = Case(32, 4, 2, 128, E4, 16, [4], [0], tail=1)
    cache, seqs = c.device(gpu)
    for seq in (seqs, F.CacheSeqs(seqs.cu_rows[:1], seqs.kv_len[:0], seqs.pages[:0])):
        q8 = torch.zeros((5, 512), dtype=torch.uint8, device=gpu)
        s = torch.full((3,), 77, dtype=torch.int32, device=gpu)
        ws = F.cache_attention_workspace(5, 4, cache, seqs, 4)
        o = blank(5, 512, gpu)
        F.llama_cache_attention(torch.zeros((5, 512), dtype=torch.bfloat16, device=gpu), cache, seq, 4, 4, o=o,
                                fq=F.FusedQuant(q8, s[0:1], ws, amax_bits=s[1:2], flags=s[2:3]))
        torch.cuda.synchronize()
        assert s.cpu().tolist() == [0, 0, F.FLAG_ZERO]
    assert (np_bits(o) == SENTINEL).all()


# ------------------------------------------------------------------ streams, graphs
def test_two_streams_with_workspaces_of_their_own(gpu):
    say("two streams")
    cs = [Case(33 + i, 8, 2, 128, E4, 16, [1, 40][i:i + 1] * 2, [900, 500]) for i in (0, 1)]
    qs = [rand_bits(c.rng, (c.rows, 1024)) for c in cs]
    devs = [c.device(gpu) for c in cs]
    qd = [strided(q, gpu, 0) for q in qs]
    want = [np_bits(F.llama_cache_attention(t, *d, 8, c.max_rows)) for t, d, c in zip(qd, devs, cs)]
    ws = [F.cache_attention_workspace(c.rows, 8, *d, c.max_rows) for c, d in zip(cs, devs)]
    outs = [[torch.empty_like(t) for _ in range(8)] for t in qd]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(8):
        for j in (0, 1):
            F.llama_cache_attention(qd[j], *devs[j], 8, cs[j].max_rows, o=outs[j][i], ws=ws[j], stream=st[j])
    torch.cuda.synchronize()
    for j in (0, 1):
        for t in outs[j]:
            assert np.array_equal(np_bits(t), want[j])


def test_captured_steps_follow_their_inputs(gpu):
    """A decode step (append, attention with the fused quantise) captured once and
    replayed token by token, lengths and inputs changed between the replays, with
    eager work and synchronisations among them."""
    say("captured steps")
    heads, kv, dh = 8, 2, 128
    c = Case(35, heads, kv, dh, E4, 16, [1, 1], [60, 9])
    e = Case(35, heads, kv, dh, E4, 16, [1, 1], [60, 9])
    (cache, seqs), (ecache, eseqs) = c.device(gpu), e.device(gpu)
    table = F.llama_rope_table(c.max_pages * 16, dh, device=gpu)
    x = torch.zeros((2, (heads + 2 * kv) * dh), dtype=torch.bfloat16, device=gpu)
    ws = F.cache_attention_workspace(2, heads, cache, seqs, 1)
    q, o = (torch.zeros((2, heads * dh), dtype=torch.bfloat16, device=gpu) for _ in "qo")
    q8, s = torch.zeros((2, heads * dh), dtype=torch.uint8, device=gpu), torch.zeros(3, dtype=torch.int32, device=gpu)
    fq = F.FusedQuant(q8, s[0:1], ws, bias_pred=s[0:1], amax_bits=s[1:2], flags=s[2:3])

    def step():
        F.llama_cache_append(x, cache, seqs, heads, table=table, q=q)
        F.llama_cache_attention(q, cache, seqs, heads, 1, o=o, fq=fq)

    step()      # writes tokens: into the eager copy too
    F.llama_cache_append(x, ecache, eseqs, heads, table=table)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    start = torch.tensor([40, 2], dtype=torch.int32, device=gpu)
    for t in range(6):
        x.copy_(strided(rand_bits(c.rng, tuple(x.shape)), gpu, 0))
        seqs.kv_len.copy_(start + t)
        g.replay()
        torch.cuda.synchronize()
        eseqs.kv_len.copy_(start + t)
        eq = F.llama_cache_append(x, ecache, eseqs, heads, table=table)
        eo = F.llama_cache_attention(eq, ecache, eseqs, heads, 1)
        rq, _, rb, ra, rf = F.fp8_quantise(eo, F.E4M3)
        assert torch.equal(q, eq) and torch.equal(o, eo) and torch.equal(q8, rq)
        assert s.cpu().tolist() == [int(rb.item()), int(ra.item()), int(rf.item())]
        for n in ("k", "v", "k_exp", "v_exp"):
            assert torch.equal(getattr(cache, n), getattr(ecache, n)), n


def test_binding_refuses_mixed_devices(gpu):
    say("mixed devices")
    c = Case(36, 4, 2, 128, E4, 16, [1], [5])
    cache, seqs = c.device(gpu)
    host = F.CacheSeqs(seqs.cu_rows.cpu(), seqs.kv_len.cpu(), seqs.pages.cpu())
    q = torch.zeros((1, 512), dtype=torch.bfloat16, device=gpu)
    with pytest.raises(ValueError):
        F.llama_cache_attention(q, cache, host, 4, 1)
    with pytest.raises(ValueError):
        F.llama_cache_attention(q.cpu(), cache, seqs, 4, 1)
    with pytest.raises(ValueError):
        F.llama_cache_read(cache, host, 1)
    with pytest.raises(ValueError):
        F.llama_cache_append(torch.zeros((1, 1024), dtype=torch.bfloat16), cache, seqs, 4)
