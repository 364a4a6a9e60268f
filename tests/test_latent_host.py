"""Host-side checks of the latent cache's entry points: sizes and refusals, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2609_17475_gb300 as jf
from paper_2609_17475_gb300 import binding as B

FAKE = ctypes.c_void_p(0x20000)   # aligned, never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x20008)
INVALID, UNSUPPORTED, SMALL = B.JF_ERR_INVALID_ARG, B.JF_ERR_UNSUPPORTED, B.JF_ERR_WORKSPACE_TOO_SMALL


def pool(**kw):
    d = dict(base=0x10000, num_pages=8, page_size=64, num_kv_heads=1, head_dim=576, group_size=64,
             format=B.JF_FMT_LATENT16)
    d.update(kw)
    return B._Pool(**d)


def test_sizes():
    L = B.lib()
    assert B.jf_kv_page_bytes_fmt(B.JF_FMT_LATENT16, 1, 256, 576) == 256 * 576 * 2
    assert B.jf_kv_page_bytes_fmt(B.JF_FMT_LATENT16, 1, 64, 320) == 64 * 320 * 2
    for hkv, d in ((2, 576), (1, 512), (1, 256), (1, 128)):
        assert B.jf_kv_page_bytes_fmt(B.JF_FMT_LATENT16, hkv, 64, d) == 0
    one = B.jf_latent_workspace_bytes(1, 16, 512, 0, 152)
    assert one >= 256 and B.jf_latent_workspace_bytes(64, 16, 512, 1, 152) >= one
    for bad in ((0, 16, 512, 0, 152), (1, 0, 512, 0, 152), (1, 1025, 512, 0, 152), (1, 16, 128, 0, 152),
                (1, 16, 512, 65, 152), (1, 16, 512, -1, 152), (65536, 16, 512, 0, 152)):
        assert B.jf_latent_workspace_bytes(*bad) == 0
    assert B.jf_latent_prefill_workspace_bytes(0, 128, 16, 152) >= 256
    for bad in ((-1, 1, 1, 152), (0, -1, 1, 152), (0, 1, 0, 152), (0, 1, 1025, 152), (0x7FFFFFFF, 1, 1, 152)):
        assert B.jf_latent_prefill_workspace_bytes(*bad) == 0
    with pytest.raises(ValueError):
        jf.latent_decode_workspace(0, 16, 512, device="cpu")
    assert L.jf_reservation_pages(1, 1, 1, 64) == 1


def append(p, **k):
    return B.lib().jf_latent_append(ctypes.byref(p), k.get("pt", FAKE), k.get("stride", 4), k.get("b", 1), FAKE, FAKE,
                                    k.get("latent", FAKE), k.get("ls", 512), k.get("rot", FAKE), k.get("rs", 64),
                                    k.get("n", 3), None, None)


def decode(p, **k):
    return B.lib().jf_latent_decode_attn(ctypes.byref(p), k.get("pt", FAKE), k.get("stride", 4), k.get("ctx", FAKE),
                                         k.get("b", 1), k.get("q", FAKE), k.get("h", 16), k.get("scale", 0.1),
                                         k.get("out", FAKE), k.get("ws", FAKE), k.get("bytes", 0), None)


def prefix(p, **k):
    off = k.get("off", [0, 2])
    arr = (ctypes.c_int32 * len(off))(*off)
    return B.lib().jf_latent_prefix_decode_attn(ctypes.byref(p), k.get("ppt", FAKE), k.get("pstride", 4), FAKE, arr,
                                                k.get("g", len(off) - 1), FAKE, 4, FAKE, k.get("b", 2), FAKE, 16, 0.1,
                                                FAKE, FAKE, k.get("bytes", 0), None)


def prefill(p, **k):
    return B.lib().jf_latent_prefill_attn(ctypes.byref(p), k.get("pt", FAKE), k.get("q", FAKE), k.get("start", 0),
                                          k.get("c", 16), k.get("h", 4), k.get("wk", FAKE), FAKE, k.get("scale", 0.1), 1,
                                          k.get("out", FAKE), k.get("ws", FAKE), k.get("bytes", 0), None)


@pytest.mark.parametrize("call", [append, decode, prefix, prefill])
@pytest.mark.parametrize("kw,expect", [
    (dict(base=None), INVALID), (dict(base=0x10008), INVALID), (dict(num_pages=0), INVALID),
    (dict(num_kv_heads=0), INVALID), (dict(num_kv_heads=2), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED),
    (dict(head_dim=128), UNSUPPORTED), (dict(page_size=32), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(format=0), UNSUPPORTED), (dict(format=8), UNSUPPORTED), (dict(num_pages=1 << 26), UNSUPPORTED),
])
def test_bad_pools_are_refused(call, kw, expect):
    assert call(pool(**kw)) == expect


def test_append_refuses_bad_arguments():
    p = pool()
    assert append(p, n=0) == 0
    for k in (dict(n=-1), dict(stride=0), dict(b=0), dict(pt=None), dict(latent=None), dict(rot=ODD), dict(latent=ODD),
              dict(ls=511), dict(ls=516), dict(ls=504), dict(rs=56), dict(rs=68)):
        assert append(p, **k) == INVALID, k


def test_decode_refuses_bad_arguments(monkeypatch):
    p = pool()
    for k in (dict(pt=None), dict(ctx=None), dict(q=None), dict(out=None), dict(ws=None), dict(q=ODD), dict(out=ODD),
              dict(ws=ctypes.c_void_p(0x20010)), dict(b=0), dict(b=65536), dict(stride=0), dict(h=0),
              dict(scale=float("nan"))):
        assert decode(p, **k) == INVALID, k
    assert decode(p, h=1025) == UNSUPPORTED
    assert decode(p) == SMALL and decode(p, bytes=255) == SMALL


def test_prefix_refuses_bad_groups():
    p = pool()
    for off in ([0, 1], [1, 2], [0, 2, 1, 2], [0, 3, 2]):
        assert prefix(p, off=off) == INVALID, off
    assert prefix(p, g=0) == INVALID and prefix(p, g=-1) == INVALID
    assert prefix(p, ppt=None) == INVALID and prefix(p, pstride=0) == INVALID
    assert prefix(p, off=[0] * 65 + [2]) == UNSUPPORTED
    assert prefix(p) == SMALL and prefix(p, off=[0, 0, 2, 2]) == SMALL


def test_prefill_refuses_bad_arguments():
    p = pool()
    for k in (dict(pt=None), dict(q=None), dict(out=None), dict(wk=None), dict(ws=None), dict(q=ODD), dict(wk=ODD),
              dict(out=ODD), dict(ws=ctypes.c_void_p(0x20010)), dict(start=-1), dict(c=-1), dict(h=0),
              dict(start=0x7FFFFFFF), dict(scale=float("nan"))):
        assert prefill(p, **k) == INVALID, k
    assert prefill(p, h=1025) == UNSUPPORTED and prefill(p) == SMALL


def test_other_entry_points_refuse_latent_pools():
    L, p = B.lib(), pool()
    r = ctypes.byref(p)
    assert L.jf_paged_decode_attn(r, FAKE, 4, FAKE, 1, FAKE, 8, 0.1, FAKE, FAKE, 1 << 30, 4, None) == UNSUPPORTED
    assert L.jf_prefill_chunk_attn(r, FAKE, FAKE, 0, 16, 8, 0.1, 1, FAKE, FAKE, 1 << 30, None) == UNSUPPORTED
    assert L.jf_kv_quantize_append(r, FAKE, 4, 1, FAKE, FAKE, FAKE, FAKE, 1, None, None) == UNSUPPORTED
    assert L.jf_kv8_append(r, FAKE, 4, 1, FAKE, FAKE, FAKE, 576, FAKE, 576, 1, None, None) == UNSUPPORTED
    # page copies take them
    assert L.jf_kv_checkpoint(r, FAKE, 1, FAKE, 64 * 576 * 2 - 1, None, None) == INVALID
    assert L.jf_kv_restore(r, FAKE, 0, FAKE, 0, None, None) == 0
    assert L.jf_kv_checkpoint(ctypes.byref(pool(head_dim=512)), FAKE, 1, FAKE, 1 << 30, None, None) == UNSUPPORTED


def test_the_binding_refuses_what_is_no_tensor_of_the_right_kind():
    p = jf.KVPool.allocate(2, 64, 1, 320, device="cpu", format=jf.JF_FMT_LATENT16)
    assert tuple(p.data.shape) == (2, 64 * 320 * 2)
    i32, bf = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 4, 320, dtype=torch.bfloat16)
    for f in (lambda: jf.jf_latent_append(p, i32, i32[0, :1], i32[0], bf[0, :, :256], bf[0, :, 256:]),
              lambda: jf.jf_latent_decode_attn(p, i32, i32[0, :1], bf, 0.1, bf[..., :256].contiguous(), i32),
              lambda: jf.jf_latent_decode_attn(p, None, i32[0, :1], bf, 0.1, bf, i32),
              lambda: jf.jf_latent_prefix_decode_attn(p, i32, i32[0, :1], [0, 1], i32, i32[0, :1], bf, 0.1, bf, i32),
              lambda: jf.jf_latent_prefill_attn(p, i32[0], bf, 0, bf, bf, 0.1, True, bf, i32)):
        with pytest.raises(TypeError):
            f()
