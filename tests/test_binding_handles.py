"""The binding's handles as Python objects: copies, pickles, assignments; and what its calls take for
a stream.  No GPU."""
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


class _Tensor:
    """What the C part reads of a CUDA tensor; its memory is never touched."""

    def __init__(self, dtype, *shape):
        self.dtype, self.shape, self.is_cuda, self.requires_grad = dtype, shape, True, False

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x20000

    def numel(self):
        return int(np.prod(self.shape))

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))


def _decode(stream, table=None):
    """A decode whose workspace is too small: refused once its arguments have been read."""
    i32, bf = torch.int32, torch.bfloat16
    p = B.KVPool(_Tensor(torch.uint8, 8, 64 * 2 * 128), 64, 1, 128, format=jf.JF_FMT_E4M3_B32)
    q = _Tensor(bf, 1, 4, 128)
    jf.jf_paged_decode_attn(p, table or _Tensor(i32, 1, 4), _Tensor(i32, 1), q, 0.1, q, _Tensor(torch.uint8, 64), 2, stream)


class _Handle:
    cuda_stream = 5


class _Int:
    def __int__(self):
        return 5


@pytest.mark.parametrize("stream", [0, 5, _Handle(), np.int64(5), np.uint64(5), _Int(), torch.tensor(5)])
def test_streams(stream):
    """A stream is an object with a handle, or anything int() takes."""
    with pytest.raises(jf.JfError) as e:
        _decode(stream)
    assert e.value.status == B.JF_ERR_WORKSPACE_TOO_SMALL


def test_what_is_no_stream():
    for stream in ("x", object(), 0.5j):
        with pytest.raises((TypeError, ValueError)):
            _decode(stream)
    with pytest.raises(OverflowError):
        _decode(-(1 << 70))


def test_tensors_without_dimensions_are_refused():
    i32, bf = torch.int32, torch.bfloat16
    with pytest.raises(ValueError):
        _decode(0, _Tensor(i32))
    p = B.KVPool(_Tensor(torch.uint8, 8, 64 * 2 * 128), 64, 1, 128, format=jf.JF_FMT_E4M3_B32)
    x, one, off = _Tensor(bf, 1, 1, 128), _Tensor(i32, 1), _Tensor(i32, 2)
    for call in (jf.jf_kv8_append, jf.jf_kv8_read):
        with pytest.raises(ValueError):
            call(p, _Tensor(i32), one, off, x, x, None, 0)
        with pytest.raises(ValueError):
            call(B.KVPool(_Tensor(torch.uint8), 64, 1, 128, format=jf.JF_FMT_E4M3_B32), _Tensor(i32, 1, 4), one, off, x, x,
                 None, 0)
