"""Rotary axes beside autograd, and at the ends of their ranges."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_in_place_is_refused_where_a_gradient_would_be_lost():
    """The call is not recorded by autograd: it does not write over rows that are part of a graph, and is seen by
    autograd's own check where it writes over what a graph has saved."""
    rope = jf.Rope(16)
    pos = torch.arange(6, dtype=torch.int32, device=DEV).view(1, 6)
    base = torch.randn(6, 2, 32, device=DEV)
    want = torch.empty_like(base)
    jf.jf_rope_axes(rope, pos, base, want)
    leaf = base.clone().requires_grad_()
    inner = leaf * 1.0
    other = torch.randn(6, 2, 32, device=DEV)
    before = other.clone()
    for args in ((leaf,), (inner,), (other, None, inner), (other, inner), (other, None, other, leaf)):
        with pytest.raises(ValueError):
            jf.jf_rope_axes(rope, pos, *args)
    assert torch.equal(leaf, base) and torch.equal(inner, base) and torch.equal(other, before)
    # rows that need a gradient may be read, and written where nothing is recorded
    got = torch.empty_like(base)
    jf.jf_rope_axes(rope, pos, inner, got)
    assert torch.equal(got, want) and not got.requires_grad
    with torch.no_grad():
        jf.jf_rope_axes(rope, pos, leaf)
    assert torch.equal(leaf, want)
    # what a graph has saved: its backward pass must not go on with other values
    w = torch.randn(32, 4, device=DEV, requires_grad=True)
    for k in (False, True):
        rows = base.clone()
        loss = (rows @ w).sum()
        if k:
            jf.jf_rope_axes(rope, pos, base, got, rows)
        else:
            jf.jf_rope_axes(rope, pos, base, rows)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    with torch.inference_mode():
        rows = base.clone()
        jf.jf_rope_axes(rope, pos, rows)
        assert torch.equal(rows, want)


def test_as_a_function_with_a_gradient():
    """Forward and inverse calls as an autograd function: the gradient is the definition's."""
    rope = jf.Rope(16, [4, 2, 2])
    g = torch.Generator(device=DEV).manual_seed(4)
    pos = torch.randint(0, 900, (3, 5), generator=g, device=DEV).int()

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            y = torch.empty_like(x)
            jf.jf_rope_axes(rope, pos, x, y)
            return y

        @staticmethod
        def backward(ctx, dy):
            dx = torch.empty_like(dy, memory_format=torch.contiguous_format)
            jf.jf_rope_axes(rope, pos, dy.contiguous(), dx, inverse=True)
            return dx
    x = torch.randn(5, 2, 32, generator=g, device=DEV, requires_grad=True)
    z = torch.randn(5, 2, 32, generator=g, device=DEV)
    (Turn.apply(x) * z).sum().backward()
    a = torch.from_numpy(rope.inv_freq.astype(np.float64)).to(DEV) * pos.double()[rope.axis.tolist()].t()     # [tokens, 8]
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    u, v = z.double()[..., :8], z.double()[..., 8:16]
    ref = torch.cat([u * c + v * s, -u * s + v * c, z.double()[..., 16:]], -1)
    assert (x.grad.double() - ref).abs().max() <= 2.0 ** -20 * z.abs().max()


def two_pi_inverse(bits=256):
    """1 / (2 pi) to `bits` bits, by Machin's formula in whole numbers."""
    one = 1 << (bits + 32)

    def arctan_inverse(n):
        total, term, k = 0, one // n, 0
        while term:
            total += (-1) ** k * (term // (2 * k + 1))
            term //= n * n
            k += 1
        return total
    pi = 4 * (4 * arctan_inverse(5) - arctan_inverse(239))
    return Fraction(one, 2 * pi)


INV = two_pi_inverse()


@pytest.mark.parametrize("inverse", [False, True])
def test_angles_at_far_positions_and_high_frequencies(inverse):
    """Frequencies from 2^-40 to just below 2^32 at the ends of the positions' range.  The angle's fraction of a turn is
    worked out exactly here; the kernel's is off by 2^-32 of a turn, and by 2^-26 in fp32 (2^-23.3 radians
    together), cosine, sine and products by a few 2^-24 more."""
    f = np.array([2.0 ** -40, 1e-3, 1.0, 3.7, 100.0, 12345.678, 2.0 ** 24 + 2, 2.0 ** 31, 2.0 ** 32 - 512, 0.5, -1.0, -77.7,
                  -3e9, 2.0 ** -126, 2.0 ** -149, 0.0], dtype=np.float32)
    pos = np.array([0, 1, -1, 2, 1 << 20, (1 << 31) - 1, -(1 << 31), 2147483001, -2000000011, 1234567891], dtype=np.int32)
    rope = jf.Rope(32, inv_freq=f)
    assert np.array_equal(rope.inv_freq, f)
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(len(pos), 3, 32, generator=g, device=DEV)
    y = torch.empty_like(x)
    jf.jf_rope_axes(rope, torch.from_numpy(pos)[None].to(DEV), x, y, inverse=inverse)
    x64, got = x.double().cpu().numpy(), y.double().cpu().numpy()
    for t, p in enumerate(pos.tolist()):
        turns = [Fraction(float(v)) * p * INV for v in f]
        a = 2 * np.pi * np.array([float(u - round(u)) for u in turns])
        c, s = np.cos(a), np.sin(a) * (-1 if inverse else 1)
        u, v = x64[t, :, :16], x64[t, :, 16:]
        ref = np.concatenate([u * c - v * s, u * s + v * c], -1)
        length = np.sqrt(u * u + v * v)
        bound = np.concatenate([length, length], -1) * 2.0 ** -21 + 2.0 ** -140
        assert (np.abs(got[t] - ref) <= bound).all(), (p, float((np.abs(got[t] - ref) / bound).max()))
