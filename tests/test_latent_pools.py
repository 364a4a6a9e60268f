"""Memory that the latent cache's calls refuse before anything is launched: a pool on the host, of another type or
shape than its fields say, tensors on another device.  No GPU: tensors are stand-ins whose memory is never touched."""
import pytest
import torch

import paper_2609_17475_gb300 as jf
from paper_2609_17475_gb300 import binding as B

I32, U8, BF = torch.int32, torch.uint8, torch.bfloat16


class Tensor:
    """What the C part reads of a tensor."""

    def __init__(self, dtype, *shape, device=0, contiguous=True):
        self.dtype, self.shape, self.device, self.contiguous = dtype, shape, device, contiguous
        self.is_cuda, self.requires_grad = device >= 0, False

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 0x20000

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def stride(self):
        out, n = [], 1
        for x in reversed(self.shape):
            out.append(n)
            n *= x
        return tuple(reversed(out))


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    """The calls ask for the current device: 0, without a driver."""
    monkeypatch.setattr(B, "_get_device", lambda: 0)
    monkeypatch.setattr(B, "_fast", None)
    yield
    monkeypatch.undo()
    B._fast = None


def pool(data, P=64, d=576, fmt=jf.JF_FMT_LATENT16):
    return jf.KVPool(data, P, 1, d, format=fmt)


def arguments(p, d=576):
    """Every entry point with everything on the GPU but what the pool says; workspaces of 64 bytes are too small, so
    that a call whose arguments pass is refused by the library instead."""
    R, table, one = d - 64, lambda: Tensor(I32, 1, 4), lambda: Tensor(I32, 1)
    rows = lambda: [p, table(), one(), Tensor(I32, 2), Tensor(BF, 3, R), Tensor(BF, 3, 64), Tensor(I32, 1), 0]  # noqa: E731
    tail = lambda: [table(), one(), Tensor(BF, 1, 4, d), 0.1, Tensor(BF, 1, 4, R), Tensor(U8, 64), 0]  # noqa: E731
    w = lambda: Tensor(BF, 4, 128, R)  # noqa: E731
    return {
        "append": (jf.jf_latent_append, rows()),
        "read": (jf.jf_latent_read, rows()),
        "decode": (jf.jf_latent_decode_attn, [p] + tail()),
        "prefix": (jf.jf_latent_prefix_decode_attn, [p, table(), one(), [0, 1]] + tail()),
        "prefill": (jf.jf_latent_prefill_attn, [p, Tensor(I32, 4), Tensor(BF, 16, 4, 192), 0, w(), w(), 0.1, True,
                                                Tensor(BF, 16, 4, 128), Tensor(U8, 64), 0]),
    }


def calls(p):
    return {name: lambda f=f, a=a: f(*a) for name, (f, a) in arguments(p).items()}


ATTEND = ["decode", "prefix", "prefill"]
ALL = ["append", "read"] + ATTEND


@pytest.mark.parametrize("name", ATTEND)
def test_a_right_pool_goes_through(name):
    with pytest.raises(jf.JfError) as e:
        calls(pool(Tensor(U8, 8, 64 * 576 * 2)))[name]()
    assert e.value.status == B.JF_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("name", ALL)
def test_a_pool_on_the_host_is_refused(name):
    """With every other tensor on the GPU."""
    for data in (Tensor(U8, 8, 64 * 576 * 2, device=-1), torch.zeros(8, 64 * 576 * 2, dtype=U8)):
        with pytest.raises(TypeError, match="pool"):
            calls(pool(data))[name]()


@pytest.mark.parametrize("name", ALL)
@pytest.mark.parametrize("data,kw,error", [
    (Tensor(torch.int8, 8, 64 * 576 * 2), {}, TypeError),
    (Tensor(BF, 8, 64 * 576), {}, TypeError),
    (Tensor(U8, 8, 64 * 576 * 2, contiguous=False), {}, TypeError),
    (Tensor(U8, 8, 64 * 320 * 2), {}, ValueError),                  # made for R = 256
    (Tensor(U8, 8, 64 * 576 * 2), dict(P=128), ValueError),
    (Tensor(U8, 8, 64 * 576 * 2 - 1), {}, ValueError),
    (Tensor(U8, 8, 64 * 576 * 2 + 16), {}, ValueError),
    (Tensor(U8, 8 * 64 * 576 * 2), {}, ValueError),
    (Tensor(U8, 8, 64, 576 * 2), {}, ValueError),
    (Tensor(U8), {}, ValueError),
    (Tensor(U8, 8, 64 * 576 * 2), dict(P=1 << 30, d=576), ValueError),
], ids=["int8", "bf16", "strided", "another R", "another page size", "a byte short", "16 bytes long", "flat", "3-D", "0-D",
        "pages past the memory"])
def test_a_pool_whose_memory_is_not_what_it_says(name, data, kw, error):
    with pytest.raises(error):
        calls(pool(data, **kw))[name]()


@pytest.mark.parametrize("name", ALL)
def test_tensors_on_another_device_are_refused(name):
    """Each of a call's tensors in turn on a second device, or on the host, the others on the current one."""
    whole = pool(Tensor(U8, 8, 64 * 576 * 2))
    f, a = arguments(whole)[name]
    for t in [whole.data] + [x for x in a if isinstance(x, Tensor)]:
        t.device = 1
        with pytest.raises(ValueError, match="another device"):
            f(*a)
        t.device, t.is_cuda = -1, False
        with pytest.raises(TypeError):
            f(*a)
        t.device, t.is_cuda = 0, True


def test_the_current_device_may_be_any(monkeypatch):
    monkeypatch.setattr(B, "_get_device", lambda: 1)
    p = pool(Tensor(U8, 8, 64 * 576 * 2, device=1))
    f, a = arguments(p)["decode"]
    with pytest.raises(ValueError, match="another device"):
        f(*a)
    for x in a:
        if isinstance(x, Tensor):
            x.device = 1
    with pytest.raises(jf.JfError) as e:
        f(*a)
    assert e.value.status == B.JF_ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("call", [jf.jf_kv8_append, jf.jf_kv8_read])
def test_an_8_bit_pool_on_the_host_is_refused(call):
    p = jf.KVPool.allocate(8, 64, 1, 128, device="cpu", format=jf.JF_FMT_E4M3_B32)
    x = Tensor(BF, 3, 1, 128)
    with pytest.raises(TypeError, match="pool"):
        call(p, Tensor(I32, 1, 4), Tensor(I32, 1), Tensor(I32, 2), x, x, None, 0)
