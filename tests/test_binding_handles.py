"""The binding's handles as Python objects: copies, pickles, assignments.  No GPU."""
import copy
import ctypes
import gc
import pickle

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from paper_2609_17475_gb300 import binding as B


def pools():
    codec = jf.Tq4Codec(128, np.ones(128), -np.ones(128))
    return [jf.KVPool.allocate(2, 64, 1, 128, device="cpu", format=f, codec=codec if f == jf.JF_FMT_TQ4 else None)
            for f in (jf.JF_FMT_AFFINE4_G64, jf.JF_FMT_TQ4, jf.JF_FMT_E4M3_B32)]


@pytest.mark.parametrize("used", [False, True])
@pytest.mark.parametrize("dup", [copy.copy, copy.deepcopy, lambda p: pickle.loads(pickle.dumps(p))])
def test_pools_copy_whether_or_not_a_call_has_used_them(dup, used):
    for p in pools():
        if used:
            p.c_struct()
        q = dup(p)
        assert torch.equal(q.data, p.data) and (q.page_size, q.format) == (p.page_size, p.format)
        c = q.c_struct()
        assert c.base == q.data.data_ptr() and c.num_pages == 2 and c.format == p.format
        if p.codec is not None:
            assert ctypes.addressof(c.tq4.contents) == ctypes.addressof(q.codec._c)
            assert list(c.tq4.contents.signs_v) [:128] == [-1] * 128


def test_pool_fields_and_properties():
    p = pools()[0]
    before = p.c_struct()
    assert p.c_struct() is before
    p.data = torch.zeros(5, p.page_bytes, dtype=torch.uint8)
    assert p.num_pages == 5 and p.c_struct().num_pages == 5 and p.c_struct().base == p.data.data_ptr()
    p.format = jf.JF_FMT_E4M3_B32
    assert p.c_struct().format == jf.JF_FMT_E4M3_B32
    for name in ("num_pages", "page_bytes"):        # worked out from data: not to be set
        with pytest.raises(AttributeError):
            setattr(p, name, 7)


class _Calls:
    """Stands for the C part of the binding: keeps what a call passes on."""

    def rope_axes(self, rope, *rest):
        self.rope = rope
        return 0


@pytest.mark.parametrize("dup", [copy.copy, copy.deepcopy, lambda p: pickle.loads(pickle.dumps(p))])
def test_rope_handles_copy(dup, monkeypatch):
    """A copy's calls read the copy's own frequencies, also when the original is gone."""
    calls = _Calls()
    monkeypatch.setattr(B, "_fast", calls)
    r = jf.Rope(32, [6, 5, 5], base=1e4)
    want, keep = r.inv_freq.copy(), ctypes.addressof(r._c)
    q = dup(r)
    del r
    gc.collect()
    jf.jf_rope_axes(q, None, None)
    assert calls.rope == ctypes.addressof(q._c) and (dup is copy.copy or calls.rope != keep)
    c = B._Rope.from_address(calls.rope)
    assert (c.rotary_dim, c.num_axes) == (32, 3) and np.array_equal(np.array(c.inv_freq[:16], dtype=np.float32), want)
