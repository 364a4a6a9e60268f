"""Host-only checks of the 8-bit cache's and the rotary axes' entry points: sizes, handles and refusals, which touch
no GPU."""
import ctypes

import numpy as np
import pytest

from paper_2609_17475_gb300 import binding as B

FAKE = 0x20000     # aligned, never dereferenced: validation fails first
I, U, W = B.JF_ERR_INVALID_ARG, B.JF_ERR_UNSUPPORTED, B.JF_ERR_WORKSPACE_TOO_SMALL


def pool(**kw):
    d = dict(base=0x10000, num_pages=8, page_size=256, num_kv_heads=2, head_dim=128, group_size=0,
             format=B.JF_FMT_E4M3_B32)
    d.update(kw)
    return B._Pool(**d)


def test_sizes():
    f = B.JF_FMT_E4M3_B32
    assert B.jf_kv_page_bytes_fmt(f, 4, 256, 256) == 2 * 4 * (256 * 256 + 4 * 8) == 256 * 2049
    assert B.jf_kv_page_bytes_fmt(f, 1, 64, 128) == 2 * (64 * 128 + 8)
    assert B.jf_kv_page_bytes_fmt(f, 1, 48, 128) == 0 and B.jf_kv_page_bytes_fmt(f, 1, 64, 64) == 0
    n = B.lib().jf_decode_weights_workspace_bytes
    base = -(-B.jf_attn_workspace_bytes(3, 24, 4, 256, 5) // 256) * 256
    assert n(3, 24, 4, 256, 5, 1000) == base + 3 * 4 * 1008 * 6 * 4
    assert n(3, 20, 4, 256, 5, 16) == -(-B.jf_attn_workspace_bytes(3, 20, 4, 256, 5) // 256) * 256 + \
        3 * 4 * 16 * 6 * 4                                    # five heads count as six
    assert n(3, 24, 5, 256, 5, 1000) == 0 and n(3, 24, 4, 256, 5, 0) == 0
    assert B.lib().jf_prefill_batch_workspace_bytes(f, 32, 8, 128, 1) == 256
    assert B.default_num_splits(1, 4, num_sms=152, format=f) == 38
    assert B.default_num_splits(2, 4, num_sms=152, format=f) == 21


@pytest.mark.parametrize("kw,expect", [
    (dict(base=None), I), (dict(base=0x10004), I), (dict(num_pages=0), I), (dict(num_kv_heads=0), I),
    (dict(head_dim=96), U), (dict(page_size=96), U), (dict(format=0, group_size=64), U), (dict(format=3), U),
])
def test_bad_pools(kw, expect):
    p, L = ctypes.byref(pool(**kw)), B.lib()
    assert L.jf_kv8_append(p, FAKE, 4, 1, FAKE, FAKE, FAKE, 256, FAKE, 256, 5, None, None) == expect
    assert L.jf_kv8_read(p, FAKE, 4, 1, FAKE, FAKE, FAKE, 256, FAKE, 256, 5, None, None) == expect
    assert L.jf_paged_decode_weights_attn(p, FAKE, 4, FAKE, 1, FAKE, 8, 0.1, FAKE, None, FAKE, 64, FAKE, 1 << 20, 4,
                                          None) == expect
    assert L.jf_kv8_evict(p, FAKE, 4, FAKE, 1, FAKE, 64, 8, 0, 0, FAKE, 4, FAKE, None, FAKE, None, None) == expect


def test_append_and_read_refuse():
    p, L = pool(), B.lib()

    def call(fn=L.jf_kv8_append, pt=FAKE, stride=4, req=1, start=FAKE, off=FAKE, k=FAKE, ks=256, v=FAKE, vs=256, n=5):
        return fn(ctypes.byref(p), pt, stride, req, start, off, k, ks, v, vs, n, None, None)
    for fn in (L.jf_kv8_append, L.jf_kv8_read):
        assert call(fn, n=0) == B.JF_OK and call(fn, n=-1) == I
        for bad in (dict(pt=None), dict(start=None), dict(off=None), dict(k=None), dict(v=None), dict(stride=0), dict(req=0),
                    dict(k=FAKE + 8), dict(v=FAKE + 2), dict(ks=255), dict(vs=252), dict(ks=248)):
            assert call(fn, **bad) == I, bad


def test_decode_weights_refuses():
    p, L = pool(), B.lib()
    big = L.jf_decode_weights_workspace_bytes(1, 8, 2, 128, 4, 64)

    def call(pt=FAKE, batch=1, hq=8, scale=0.1, w_in=None, w=FAKE, stride=64, ws=FAKE, wsb=big - 1, splits=4):
        return L.jf_paged_decode_weights_attn(ctypes.byref(p), pt, 4, FAKE, batch, FAKE, hq, scale, FAKE, w_in, w, stride,
                                              ws, wsb, splits, None)
    assert call() == W
    assert call(hq=18) == U and call(hq=7) == I and call(batch=0) == I and call(splits=0) == I and call(pt=None) == I
    assert call(w=None) == I and call(w=FAKE + 2) == I and call(w_in=FAKE + 1) == I and call(stride=0) == I
    assert call(scale=float("nan")) == I and call(ws=FAKE + 16) == I


def test_decode_and_prefill_take_the_format_and_the_others_refuse():
    p, L = ctypes.byref(pool()), B.lib()
    assert L.jf_paged_decode_attn(p, FAKE, 4, FAKE, 1, FAKE, 8, 0.1, FAKE, FAKE, 100, 4, None) == W
    assert L.jf_paged_decode_attn(p, FAKE, 4, FAKE, 1, FAKE, 18, 0.1, FAKE, FAKE, 1 << 20, 4, None) == U
    assert L.jf_prefill_chunk_attn(p, FAKE, FAKE, 0, 16, 8, 0.1, 1, FAKE, FAKE, 0, None) == W
    assert L.jf_prefill_chunk_attn(p, FAKE, FAKE, 0, 0, 8, 0.1, 1, FAKE, FAKE, 256, None) == B.JF_OK
    for n in (1, 2, 4):
        assert L.jf_paged_verify_attn(p, FAKE, 4, FAKE, 1, FAKE, n, 8, 0.1, FAKE, FAKE, 1 << 20, 4, None) == U
    assert L.jf_paged_decode_append_attn(p, FAKE, 4, FAKE, 1, FAKE, FAKE, FAKE, 8, 0.1, FAKE, FAKE, 1 << 20, 4, None) == U
    assert L.jf_paged_decode_attn_noalloc(p, FAKE, 4, FAKE, 1, FAKE, 8, 0.1, FAKE, 4, None, None) == U
    assert L.jf_kv_quantize_append(p, FAKE, 4, 1, FAKE, FAKE, FAKE, FAKE, 5, None, None) == U
    pb = B.jf_kv_page_bytes_fmt(B.JF_FMT_E4M3_B32, 2, 256, 128)
    assert L.jf_kv_checkpoint(p, FAKE, 3, FAKE, 3 * pb - 1, None, None) == I


def test_evict_refuses():
    p, L = pool(), B.lib()

    def call(pt=FAKE, batch=1, w=FAKE, stride=64, budget=8, sinks=0, recent=0, dst=FAKE, dstride=4, ctx=FAKE, kept=FAKE):
        return L.jf_kv8_evict(ctypes.byref(p), pt, 4, FAKE, batch, w, stride, budget, sinks, recent, dst, dstride, ctx, None,
                              kept, None, None)
    for bad in (dict(pt=None), dict(batch=0), dict(batch=65536), dict(w=None), dict(w=FAKE + 2), dict(stride=0),
                dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=5, recent=4), dict(dst=None), dict(dstride=0),
                dict(ctx=None), dict(kept=None), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1)):
        assert call(**bad) == I, bad


def test_rope_handles_and_refusals():
    r = B.Rope(32, [6, 5, 5], base=1e4, layout="interleaved")
    assert r.axis.tolist() == [0, 1, 2] * 5 + [0]
    assert np.array_equal(r.inv_freq, (1e4 ** (-np.arange(16) / 16)).astype(np.float32))
    assert B.Rope(32, [6, 5, 5]).axis.tolist() == [0] * 6 + [1] * 5 + [2] * 5
    assert B.Rope(16, [4, 2, 2], axis=[2, 1, 0, 0, 1, 2, 0, 1]).axis.tolist() == [2, 1, 0, 0, 1, 2, 0, 1]
    for bad in (dict(rotary_dim=24), dict(rotary_dim=272), dict(rotary_dim=32, sections=[8, 4]),
                dict(rotary_dim=32, sections=[4, 4, 4, 4]), dict(rotary_dim=32, sections=[17, -1]),
                dict(rotary_dim=32, layout="x"), dict(rotary_dim=32, pairing="x"),
                dict(rotary_dim=32, inv_freq=np.ones(8)), dict(rotary_dim=16, axis=[0] * 7 + [1])):
        with pytest.raises(ValueError):
            B.Rope(**bad)
    L = B.lib()
    rows = lambda **kw: B._RopeRows(**{**dict(in_=FAKE, out=FAKE, in_token_stride=256, in_head_stride=64,
                                              out_token_stride=256, out_head_stride=64, num_heads=4), **kw})
    none = B._RopeRows()

    def call(rope=r, pos=FAKE, stride=9, n=9, d=64, q=None, k=none, dtype=0):
        return L.jf_rope_axes(ctypes.byref(rope._c) if hasattr(rope, "_c") else ctypes.byref(rope), pos, stride, n, d,
                              ctypes.byref(rows() if q is None else q), ctypes.byref(k), dtype, 0, None)
    assert call(n=0) == B.JF_OK and call(q=none) == B.JF_OK          # nothing to turn
    assert call(pos=None) == I and call(n=-1) == I and call(stride=-1) == I
    assert call(d=16) == U and call(d=72) == U and call(d=528) == U and call(dtype=3) == U
    for bad in (dict(in_=None), dict(out=None), dict(in_=FAKE + 8), dict(in_token_stride=255), dict(out_head_stride=4),
                dict(num_heads=-1), dict(out_token_stride=512)):     # the last: in place, but to other rows
        assert call(q=rows(**bad)) == I, bad
        assert call(q=none, k=rows(**bad)) == I, bad
    assert call(q=rows(in_token_stride=258), dtype=2) == I          # fp32 rows start on 4 elements
    for field, value, status in (("rotary_dim", 40, U), ("rotary_dim", 0, U), ("pairing", 2, I), ("num_axes", 0, I),
                                 ("num_axes", 4, I)):
        c = B._Rope.from_buffer_copy(r._c)
        setattr(c, field, value)
        assert call(rope=c) == status
    c = B._Rope.from_buffer_copy(r._c)
    c.axis[3] = 3
    assert call(rope=c) == I
    for f in (float("nan"), float("inf"), 2.0 ** 32):
        c = B._Rope.from_buffer_copy(r._c)
        c.inv_freq[15] = f
        assert call(rope=c) == I


def test_positions_of_the_session_example():
    import importlib.util
    import os
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "long_session.py")
    spec = importlib.util.spec_from_file_location("long_session", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    p = m.positions(2000, 16)
    assert p[:, 300].tolist() == [300] * 3 and p[:, 1024 + 17].tolist() == [1024, 1025, 1025]
