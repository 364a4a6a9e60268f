"""The binding's handles as Python objects: copies, pickles, assignments.  No GPU."""
import copy
import ctypes
import pickle

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf


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
