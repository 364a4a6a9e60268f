"""Rotary axes beside autograd, and at the ends of their ranges."""
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
