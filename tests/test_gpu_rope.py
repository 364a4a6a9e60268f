"""Rotary positions with several axes on the GPU against the fp64 definition."""
import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import rope as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
# half a unit in the last place of each type, of the value at most
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def check(x, y, ref, dtype):
    """One rounding of the result, and errors of a few 2^-24 of the pair's length in the fp32 products and the
    cosines (angles are off by at most 2^-32 of a turn, their fp32 form by 2^-25 of a half turn)."""
    length = np.abs(x).max(-1, keepdims=True) * 2.0 ** 0.5
    bound = np.abs(ref) * UNIT[dtype] * 1.01 + length * 2.0 ** -21 + 2.0 ** -25
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= bound).all(), float((err - bound).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("n,hq,hkv,d,rot,sections,layout,pairing", [
    (1, 24, 4, 256, 64, [8, 12, 12], "interleaved", "half"),
    (33, 8, 2, 128, 128, [24, 20, 20], "sectioned", "half"),
    (7, 3, 1, 80, 48, [24], "sectioned", "adjacent"),
    (301, 5, 5, 112, 96, [20, 28], "interleaved", "adjacent"),
    (2, 1, 0, 16, 16, [0, 4, 4], "sectioned", "half"),
    (64, 16, 8, 512, 256, [44, 42, 42], "interleaved", "half"),
])
def test_turns_like_the_definition(dtype, n, hq, hkv, d, rot, sections, layout, pairing):
    rng = np.random.default_rng(n * 7 + rot)
    rope = jf.Rope(rot, sections, base=1e6, layout=layout, pairing=pairing)
    assert rope.axis.tolist() == R.axes_of(sections, layout)
    # near, negative and far positions
    pos = rng.integers(-300, 300000, (len(sections), n)).astype(np.int32)
    if n > 2:
        pos[:, 0], pos[:, 1] = 2 ** 31 - 1, -2 ** 31
    p = torch.from_numpy(pos).to(DEV)
    x = [torch.from_numpy(rng.standard_normal((n, h, d))).to(dtype).to(DEV) for h in (hq, hkv)]
    for inverse in (False, True):
        y = [torch.full_like(t, float("nan")) for t in x]
        jf.jf_rope_axes(rope, p, x[0], y[0], x[1] if hkv else None, y[1] if hkv else None, inverse=inverse)
        for a, b, h in zip(x, y, (hq, hkv)):
            if h:
                a64 = a.double().cpu().numpy()
                check(a64, b, R.rotate(a64, pos, rope.axis, rope.inv_freq, pairing, inverse), dtype)
                assert torch.equal(a[..., rot:], b[..., rot:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_strides_and_in_place(dtype):
    """Heads of one fused projection, outputs into a wider buffer, and in place: the bits of the plain call."""
    rng = np.random.default_rng(1)
    n, hq, hkv, d = 19, 4, 2, 128
    rope = jf.Rope(64, [12, 10, 10], pairing="adjacent")
    pos = torch.from_numpy(rng.integers(0, 9000, (3, n + 5)).astype(np.int32)).to(DEV)[:, :n]
    qkv = torch.randn(n, hq + 2 * hkv, d, device=DEV).to(dtype)
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    want = [torch.empty(n, h, d, dtype=dtype, device=DEV) for h in (hq, hkv)]
    jf.jf_rope_axes(rope, pos, q.contiguous(), want[0], k.contiguous(), want[1])
    wide = torch.zeros(n, hkv + 1, d + 16, dtype=dtype, device=DEV)
    got_q = torch.empty(hq, n, d, dtype=dtype, device=DEV).permute(1, 0, 2)     # heads outermost
    jf.jf_rope_axes(rope, pos, q, got_q, k, wide[:, 1:, :d])
    assert torch.equal(got_q, want[0]) and torch.equal(wide[:, 1:, :d], want[1])
    assert not wide[:, 0].any() and not wide[:, :, d:].any()
    rest = qkv[:, hq + hkv:].clone()
    jf.jf_rope_axes(rope, pos, q, None, k, None)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, hq + hkv:], rest)


def test_gradient_against_differences():
    """d/dx of <z, rope(x)> is the inverse call on z: against the definition and central differences
    (the map is linear, so a difference is off by rounding alone: fp32 sums of 2 n h d terms)."""
    g = torch.Generator(device=DEV).manual_seed(2)
    n, h, d = 5, 2, 64
    rope = jf.Rope(32, [6, 5, 5], layout="interleaved")
    pos = torch.randint(-50, 5000, (3, n), generator=g, device=DEV).int()
    x, z = (torch.randn(n, h, d, generator=g, device=DEV) for _ in range(2))
    grad = torch.empty_like(z)
    jf.jf_rope_axes(rope, pos, z, grad, inverse=True)
    z64 = z.double().cpu().numpy()
    check(z64, grad, R.rotate(z64, pos.cpu().numpy(), rope.axis, rope.inv_freq, "half", True), torch.float32)

    def value(t):
        y = torch.empty_like(t)
        jf.jf_rope_axes(rope, pos, t, y)
        return float((y.double() * z.double()).sum())
    for i, j, c in ((0, 0, 0), (1, 1, 17), (4, 0, 31), (3, 1, 40)):
        e = torch.zeros_like(x)
        e[i, j, c] = 0.5
        # each element of y is off by 2^-22 of |x| <= 6 at most, summed over n h d = 640 of them with |z| <= 6
        assert abs((value(x + e) - value(x - e)) - float(grad[i, j, c])) <= 2 * 640 * 36 * 2.0 ** -22


def test_forward_then_inverse_and_far_positions_keep_their_angle():
    """A far position turns like the same angle near zero: with a frequency of 2 pi / 1024 positions p and
    p + 1024 m agree, up to the fp32 frequency's own error at that distance."""
    x = torch.randn(1, 1, 16, device=DEV).repeat(2, 1, 1)
    f = np.full(8, 2 * np.pi / 1024)
    rope = jf.Rope(16, inv_freq=f)
    far = 5 + 1024 * 2 ** 20
    y = torch.empty_like(x)
    pos = torch.tensor([[far, far]], dtype=torch.int32, device=DEV)
    jf.jf_rope_axes(rope, pos, x, y)
    ref = R.rotate(x.double().cpu().numpy(), pos.cpu().numpy(), rope.axis, rope.inv_freq, "half")
    check(x.double().cpu().numpy(), y, ref, torch.float32)
    back = torch.empty_like(x)
    jf.jf_rope_axes(rope, pos, y, back, inverse=True)
    assert (back - x).abs().max() <= 2.0 ** -20 * x.abs().max()


def test_no_tokens_other_streams_and_refusals():
    rope = jf.Rope(16)
    pos = torch.zeros(1, 0, dtype=torch.int32, device=DEV)
    jf.jf_rope_axes(rope, pos, torch.empty(0, 2, 32, device=DEV))
    pos = torch.arange(6, dtype=torch.int32, device=DEV).view(1, 6)
    x = torch.randn(6, 2, 32, device=DEV)
    want, got = torch.empty_like(x), torch.empty_like(x)
    jf.jf_rope_axes(rope, pos, x, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        jf.jf_rope_axes(rope, pos, x, got)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    with pytest.raises(ValueError):
        jf.jf_rope_axes(rope, pos, None)
    with pytest.raises(ValueError):
        jf.jf_rope_axes(rope, pos, x[:5])
    with pytest.raises(TypeError):
        jf.jf_rope_axes(rope, pos.long(), x)
    with pytest.raises(TypeError):
        jf.jf_rope_axes(rope, pos, x.double())
    with pytest.raises(ValueError):
        jf.jf_rope_axes(rope, pos, torch.randn(6, 32, 2, device=DEV).transpose(1, 2))   # channels apart
    with pytest.raises(jf.JfError) as e:   # rows that do not start on 16 bytes
        jf.jf_rope_axes(rope, pos, torch.randn(6, 2, 33, device=DEV)[..., 1:])
    assert e.value.status == jf.binding.JF_ERR_INVALID_ARG
    with pytest.raises(jf.JfError) as e:   # in place, but to other rows
        b = torch.randn(12, 2, 32, device=DEV)
        jf.jf_rope_axes(rope, pos, b[:6], b[::2])
    assert e.value.status == jf.binding.JF_ERR_INVALID_ARG
    with pytest.raises(jf.JfError) as e:   # more rotated channels than there are
        jf.jf_rope_axes(jf.Rope(64), pos, x)
    assert e.value.status == jf.binding.JF_ERR_UNSUPPORTED
