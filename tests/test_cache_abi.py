"""Refusals of the paged key/value cache calls, on the host (no GPU needed): the
C entry points reject bad arguments before they would launch anything, and the
binding rejects tensors of wrong types, shapes and devices."""
import ctypes

import pytest
import torch

from paper_2309_17224_amd import fp8lin as F

FAKE, A8, ODD = 0x100000, 0x100008, 0x100001   # never dereferenced


@pytest.fixture(scope="module")
def L():
    return F.lib()


def cache(**kw):
    d = dict(k=FAKE, v=FAKE, k_exp=FAKE, v_exp=FAKE, n_pages=8, n_kv_heads=2, d_head=128, page_size=16, fmt=F.E4M3)
    d.update(kw)
    return F.CacheStruct(*[d[f[0]] for f in F.CacheStruct._fields_])


def seqs(**kw):
    d = dict(cu_rows=FAKE, kv_len=FAKE, pages=FAKE, n_seqs=3, max_pages=4, ld_pages=4)
    d.update(kw)
    return F.SeqsStruct(*[d[f[0]] for f in F.SeqsStruct._fields_])


BAD_CACHES = [
    (dict(k=None), F.EINVAL), (dict(v=None), F.EINVAL), (dict(k_exp=None), F.EINVAL), (dict(v_exp=None), F.EINVAL),
    (dict(k=A8), F.EINVAL), (dict(v=A8), F.EINVAL), (dict(k_exp=ODD), F.EINVAL), (dict(v_exp=A8), F.EINVAL),
    (dict(n_pages=0), F.EINVAL), (dict(n_pages=-1), F.EINVAL), (dict(n_pages=1 << 31), F.ENOTSUP),
    (dict(n_kv_heads=0), F.EINVAL), (dict(n_kv_heads=5000), F.ENOTSUP), (dict(d_head=96), F.ENOTSUP),
    (dict(d_head=256), F.ENOTSUP), (dict(page_size=8), F.EINVAL), (dict(page_size=48), F.EINVAL),
    (dict(page_size=2048), F.EINVAL), (dict(page_size=0), F.EINVAL), (dict(page_size=-16), F.EINVAL),
    (dict(fmt=F.E4_A), F.ENOTSUP), (dict(fmt=F.E5_A), F.ENOTSUP), (dict(fmt=4), F.EINVAL), (dict(fmt=-1), F.EINVAL),
]
BAD_SEQS = [
    (dict(cu_rows=None), F.EINVAL), (dict(kv_len=None), F.EINVAL), (dict(pages=None), F.EINVAL),
    (dict(cu_rows=ODD), F.EINVAL), (dict(kv_len=ODD), F.EINVAL), (dict(pages=ODD), F.EINVAL),
    (dict(n_seqs=-1), F.EINVAL), (dict(n_seqs=(1 << 20) + 1), F.ENOTSUP), (dict(max_pages=-1), F.EINVAL),
    (dict(ld_pages=3), F.EINVAL), (dict(max_pages=1 << 27, ld_pages=1 << 27), F.ENOTSUP),
]


def calls(L, c, s, rows=5, heads=4):
    """Status of each entry point with otherwise good arguments."""
    pc, ps = (None if x is None else ctypes.addressof(x) for x in (c, s))
    dh = 128 if c is None else max(c.d_head, 1)
    nk = 2 if c is None else max(c.n_kv_heads, 1)
    return [
        L.llama_cache_append(FAKE, rows, (heads + 2 * nk) * dh, heads, pc, ps, FAKE, 1 << 31, FAKE, heads * dh, None),
        L.llama_cache_read(pc, ps, rows, FAKE, nk * dh, FAKE, nk * dh, None),
        L.llama_cache_attention(FAKE, rows, heads * dh, heads, pc, ps, rows, 0, FAKE, heads * dh, 0, 0, None, None,
                                None, None, None, 0, FAKE, 1 << 40, None),
    ]


@pytest.mark.parametrize("kw,status", BAD_CACHES, ids=lambda x: str(x))
def test_bad_caches(L, kw, status):
    assert calls(L, cache(**kw), seqs(), heads=2 * max(1, kw.get("n_kv_heads", 2))) == [status] * 3


@pytest.mark.parametrize("kw,status", BAD_SEQS, ids=lambda x: str(x))
def test_bad_sequences(L, kw, status):
    assert calls(L, cache(), seqs(**kw)) == [status] * 3


def test_null_structs_and_rows(L):
    assert calls(L, None, seqs()) == [F.EINVAL] * 3
    assert calls(L, cache(), None) == [F.EINVAL] * 3
    assert calls(L, cache(), seqs(), rows=-1) == [F.EINVAL] * 3
    assert calls(L, cache(), seqs(), rows=(1 << 27) + 1) == [F.ENOTSUP] * 3


def test_nothing_to_do_launches_nothing(L):
    """No rows, or no sequences: success without a GPU."""
    assert calls(L, cache(), seqs(), rows=0) == [F.OK] * 3
    assert calls(L, cache(), seqs(n_seqs=0, cu_rows=None, kv_len=None, pages=None)) == [F.OK] * 3
    c, s = cache(), seqs()
    assert L.llama_cache_attention(FAKE, 5, 512, 4, ctypes.addressof(c), ctypes.addressof(s), 0, 0, FAKE, 512, 0, 0,
                                   None, None, None, None, None, 0, FAKE, 1 << 40, None) == F.OK


def test_append_rejects(L):
    c, s = cache(), seqs()
    pc, ps = ctypes.addressof(c), ctypes.addressof(s)

    def f(qkv=FAKE, rows=5, ld=1024, heads=4, table=FAKE, tlen=64, q=FAKE, ldq=512):
        return L.llama_cache_append(qkv, rows, ld, heads, pc, ps, table, tlen, q, ldq, None)

    for kw in (dict(qkv=None), dict(qkv=A8), dict(ld=1016), dict(ld=1028), dict(heads=3), dict(heads=0),
               dict(heads=-4), dict(heads=65538), dict(table=A8), dict(tlen=63), dict(tlen=-1), dict(q=A8),
               dict(ldq=504), dict(ldq=516)):
        assert f(**kw) == F.EINVAL, kw


def test_read_rejects(L):
    c, s = cache(), seqs()
    pc, ps = ctypes.addressof(c), ctypes.addressof(s)

    def f(k=FAKE, ldk=256, v=FAKE, ldv=256):
        return L.llama_cache_read(pc, ps, 5, k, ldk, v, ldv, None)

    for kw in (dict(k=None, v=None), dict(k=A8), dict(v=A8), dict(ldk=248), dict(ldv=248), dict(ldk=260),
               dict(ldv=260)):
        assert f(**kw) == F.EINVAL, kw


def test_attention_rejects(L):
    c, s = cache(), seqs()
    pc, ps = ctypes.addressof(c), ctypes.addressof(s)
    need = L.llama_cache_attention_ws_bytes(5, 4, pc, ps, 5)

    def f(q=FAKE, ldq=512, heads=4, max_rows=5, window=0, o=FAKE, ldo=512, fmt=0, margin=0, bias=None, q8=None,
          ldq8=512, ws=FAKE, wsb=1 << 30):
        return L.llama_cache_attention(q, 5, ldq, heads, pc, ps, max_rows, window, o, ldo, fmt, margin, None, bias,
                                       None, None, q8, ldq8, ws, wsb, None)

    for kw in (dict(q=None), dict(o=None), dict(q=A8), dict(o=A8), dict(ldq=504), dict(ldo=504), dict(ldq=516),
               dict(ldo=516), dict(heads=3), dict(heads=0), dict(max_rows=-1), dict(window=-1),
               dict(q8=FAKE), dict(q8=FAKE, bias=FAKE, fmt=9), dict(q8=FAKE, bias=FAKE, margin=1 << 20),
               dict(q8=ODD, bias=FAKE), dict(q8=FAKE, bias=ODD), dict(q8=FAKE, bias=FAKE, ldq8=504),
               dict(q8=FAKE, bias=FAKE, ws=None), dict(q8=FAKE, bias=FAKE, wsb=4)):
        assert f(**kw) == F.EINVAL, kw
    if need:
        assert f(ws=None) == F.EINVAL and f(ws=A8) == F.EINVAL and f(wsb=need - 1) == F.EINVAL


def test_workspace_bytes(L):
    c = cache()
    pc = ctypes.addressof(c)
    small, big = seqs(), seqs(n_seqs=1, max_pages=1 << 16, ld_pages=1 << 16)

    def f(rows=5, heads=4, pc=pc, s=small, m=5):
        return L.llama_cache_attention_ws_bytes(rows, heads, pc, ctypes.addressof(s), m)

    assert f(rows=0) == f(rows=-1) == f(heads=3) == f(m=0) == f(pc=None) == 0
    assert f(rows=1, s=big, m=1) < 1 << 28       # one token over a million: megabytes, not the scores


def host_cache(**kw):
    d = dict(n_pages=4, n_kv_heads=2, d_head=64, page_size=16, fmt=F.E4M3, device="cpu")
    d.update(kw)
    return F.KVCache(**d)


def host_seqs():
    i = dict(dtype=torch.int32)
    return F.CacheSeqs(torch.tensor([0, 2], **i), torch.tensor([2], **i), torch.zeros((1, 2), **i))


def test_binding_refuses_host_tensors():
    c, s = host_cache(), host_seqs()
    x = torch.zeros((2, 4 * 64 + 4 * 64), dtype=torch.bfloat16)
    for call in (lambda: F.llama_cache_append(x, c, s, 4), lambda: F.llama_cache_read(c, s, 2),
                 lambda: F.llama_cache_attention(x[:, :256], c, s, 4, 2)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()


def test_binding_refuses_types_and_shapes():
    c, s = host_cache(), host_seqs()
    x = torch.zeros((2, 512), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        F.llama_cache_append(x.float(), c, s, 4)
    with pytest.raises(ValueError):
        F.llama_cache_append(x, c, s, 6)                               # columns of other heads
    with pytest.raises(ValueError):
        F.llama_cache_append(x, c, s, 4, q=x[:1, :256])                # too few rows
    with pytest.raises(TypeError):
        F.llama_cache_read(c, s, 2, k=torch.zeros((2, 128)))
    with pytest.raises(ValueError):
        F.llama_cache_read(c, s, 2, v=torch.zeros((2, 64), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        F.llama_cache_attention(x, c, s, 4, 2)
    with pytest.raises(ValueError):
        host_cache(k=torch.zeros((4, 2, 16, 32), dtype=torch.uint8))
    with pytest.raises(TypeError):
        host_cache(v=torch.zeros((4, 2, 1, 64, 16), dtype=torch.bfloat16))
    i = dict(dtype=torch.int32)
    with pytest.raises(TypeError):
        F.CacheSeqs(torch.zeros(2, **i), torch.zeros(1, **i), torch.zeros((1, 2)))
    with pytest.raises(TypeError):
        F.CacheSeqs(torch.zeros(2), torch.zeros(1, **i), torch.zeros((1, 2), **i))
    with pytest.raises(ValueError):
        F.CacheSeqs(torch.zeros(3, **i), torch.zeros(1, **i), torch.zeros((1, 2), **i))
    with pytest.raises(ValueError):
        F.CacheSeqs(torch.zeros(2, **i), torch.zeros(1, **i), torch.zeros((2, 2), **i))
    with pytest.raises(ValueError):                                    # rows of the table not contiguous
        F.CacheSeqs(torch.zeros(3, **i), torch.zeros(2, **i), torch.zeros((4, 2), **i).t()[:, ::2])
