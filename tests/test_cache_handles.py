"""KVCache and CacheSeqs describe their tensors to the C calls by address: what they describe
cannot be replaced behind the description (on the host; nothing is launched)."""
import copy

import pytest
import torch

from paper_2309_17224_amd import fp8lin as F


def cache(fmt=F.E4M3):
    return F.KVCache(3, 2, 64, 16, fmt, "cpu")


def seqs():
    i = dict(dtype=torch.int32)
    return F.CacheSeqs(torch.tensor([0, 2, 3], **i), torch.tensor([2, 9], **i), torch.zeros((2, 4), **i))


def described(x):
    """Each attribute and its value in the struct."""
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    names = [f[0] for f in type(x._c)._fields_]
    return {n: (getattr(x._c, n), at(getattr(x, n)) if torch.is_tensor(getattr(x, n, 0)) else getattr(x, n, None))
            for n in names if n != "ld_pages"}


@pytest.mark.parametrize("x", [cache(), cache(F.E5M2), cache(F.CACHE_BF16), seqs()], ids=["e4m3", "e5m2", "bf16", "seqs"])
def test_attributes_cannot_leave_the_struct(x):
    before = described(x)
    assert all(a == b for a, b in before.values())
    for name in before:
        old = getattr(x, name)
        for new in (old.clone(), old.view(torch.int8)) if torch.is_tensor(old) else (-1, 1.5, torch.zeros(1)):
            with pytest.raises(AttributeError, match=name):
                setattr(x, name, new)
        with pytest.raises(AttributeError):
            delattr(x, name)
        assert getattr(x, name) is old
    for name in ("device", "_c", "_ref", "_dev"):
        with pytest.raises(AttributeError):
            setattr(x, name, None)
    assert described(x) == before
    x.note = "its owner's"             # other attributes are the user's
    del x.note


def test_contents_change_in_place():
    s = seqs()
    p = s._c.kv_len
    s.kv_len.copy_(torch.tensor([4, 10], dtype=torch.int32))
    s.kv_len += 1                            # in place: sets the tensor that is there
    s.kv_len[0] = 7
    assert s._c.kv_len == p == s.kv_len.data_ptr() and s.kv_len.tolist() == [7, 11]
    with pytest.raises(AttributeError):
        s.kv_len = s.kv_len + 1
    assert s._c.kv_len == p == s.kv_len.data_ptr() and s.kv_len.tolist() == [7, 11]


def test_shallow_copy_describes_the_same_tensors():
    s = seqs()
    t = copy.copy(s)
    assert t._c.kv_len == s.kv_len.data_ptr() and t.kv_len is s.kv_len
    with pytest.raises(AttributeError):
        t.kv_len = s.kv_len.clone()
