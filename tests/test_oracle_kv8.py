"""The 8-bit cache's and the rotary axes' oracles, pinned on the CPU."""
import numpy as np
import pytest
import torch

from oracle import kv8 as O
from oracle import rope as R
from tests import kv8_cases as C


def test_codes_equal_torch_e4m3():
    """Every code's value, and the rounding of values around every code and every midpoint."""
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(v), np.isnan(O.VALUES))
    fine = ~np.isnan(v)
    assert np.array_equal(v[fine], O.VALUES[fine])
    pos = O.VALUES[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    y = np.concatenate([pos, mid, np.nextafter(mid.astype(np.float32), 0), mid * (1 + 2.0 ** -20)])
    y = np.concatenate([y, -y]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O.round_codes(y.astype(np.float64)), want)
    assert np.array_equal(O.round_codes(np.array([1e9, -1e9, np.inf, np.nan])), [126, 254, 126, 127])


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0001, 1), (224.0, -1), (1.75, -8), (1.7500001, -7),
                                   (0.0, -40), (1e-30, -40), (1e30, 40)])
def test_exponent(top, e):
    x = np.zeros((3, 4))
    x[1, 2] = -top
    assert O.exponent(x) == e
    x[0, 0], x[2, 3] = np.nan, np.inf       # not counted
    assert O.exponent(x) == e


def test_append_in_parts_keeps_the_scale_and_the_values():
    """Row by row or at once: the same scales, and values apart by less than the smallest code's step."""
    rng = np.random.default_rng(3)
    L = O.Layout(2, 64, 128)
    k, v = C.rows(rng, 100, 2, 128), C.rows(rng, 100, 2, 128)
    k[37] *= 64
    one, two = O.new_pool(L, 2), O.new_pool(L, 2)
    O.append(one, L, [[1, 0]], [0], [0, 100], k, v)
    for i in range(100):
        O.append(two, L, [[1, 0]], [i], [0, 1], k[i:i + 1], v[i:i + 1])
    assert np.array_equal(L.views(one)[1], L.views(two)[1])
    a, b = O.read(one, L, [1, 0], 100), O.read(two, L, [1, 0], 100)
    s = np.repeat(L.views(one)[1][[1, 0]], 32, -1).transpose(1, 0, 3, 2).reshape(2, 128, 2)[:, :100, :, None]
    for kind in range(2):
        assert (np.abs(a[kind] - b[kind]) <= 2.0 ** -9 * s[kind]).all()
        x = (k, v)[kind]
        assert (np.abs(a[kind] - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * s[kind])).all()


def test_attend_equals_torch_sdpa():
    rng = np.random.default_rng(4)
    k, v, q = rng.standard_normal((50, 2, 16)), rng.standard_normal((50, 2, 16)), rng.standard_normal((5, 6, 16))
    out, w, _ = O.attend(k, v, q, 0.25, limit=[46, 47, 48, 49, 50])
    t = lambda x: torch.from_numpy(x).permute(1, 0, 2)
    mask = torch.arange(50)[None] < torch.arange(46, 51)[:, None]
    ref = torch.nn.functional.scaled_dot_product_attention(
        t(q), t(k).repeat_interleave(3, 0), t(v).repeat_interleave(3, 0), attn_mask=mask, scale=0.25)
    assert np.allclose(out, ref.permute(1, 0, 2).numpy(), atol=1e-12)
    assert np.allclose(w.sum(-1), 1)
    assert not O.attend(k[:0], v[:0], q, 0.25)[0].any()


def test_keep():
    w = np.array([0, 5, 1, 5, np.nan, 2, 5, -np.inf, 0.0, -0.0], dtype=np.float32)
    assert O.keep(w, 2, 0, 0).tolist() == [1, 3]              # equal weights: the lower position
    assert O.keep(w, 4, 1, 1).tolist() == [0, 1, 3, 9]
    assert O.keep(w, 5, 0, 0).tolist() == [1, 2, 3, 5, 6]
    assert O.keep(w, 6, 0, 0).tolist() == [0, 1, 2, 3, 5, 6]
    assert O.keep(w, 9, 0, 0).tolist() == [0, 1, 2, 3, 5, 6, 7, 8, 9]   # NaN goes first
    assert O.keep(w, 20, 3, 3).tolist() == list(range(10))


def test_rotation_turns_and_its_inverse_is_its_transpose():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 3, 32))
    pos = rng.integers(-9, 9, (2, 4))
    axis = R.axes_of([5, 3], "interleaved")
    assert axis == [0, 1, 0, 1, 0, 1, 0, 0]
    assert R.axes_of([5, 3], "sectioned") == [0] * 5 + [1] * 3
    f = np.float32(1e4) ** (-np.arange(8, dtype=np.float32) / 8)
    for pairing in ("half", "adjacent"):
        y = R.rotate(x, pos, axis, f, pairing)
        assert np.allclose(R.rotate(y, pos, axis, f, pairing, inverse=True), x)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 16:], x[..., 16:])
        z = rng.standard_normal(x.shape)
        # <R x, z> = <x, R^T z>
        assert np.isclose((y * z).sum(), (x * R.rotate(z, pos, axis, f, pairing, inverse=True)).sum())
        # against complex multiplication
        a, b = (slice(0, 8), slice(8, 16)) if pairing == "half" else (slice(0, 16, 2), slice(1, 16, 2))
        ang = pos[axis].T.astype(np.float64) * f
        c = (x[..., a] + 1j * x[..., b]) * np.exp(1j * ang)[:, None]
        assert np.allclose(y[..., a], c.real) and np.allclose(y[..., b], c.imag)
