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
