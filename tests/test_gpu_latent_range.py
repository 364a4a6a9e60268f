"""Latent prefill on the GPU over the range of its values: heads and positions of any magnitude, positions that
draw most of the weight and hold next to nothing, latents of zero; against the fp64 definition."""
import math

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import latent as O
from tests import latent_cases as T
from tests.latent_cases import f64, gpu, ints

pytestmark = pytest.mark.gpu
RANGE = 16   # JF_DEV_ERR_RANGE


def weights(rng, H, R):
    return T.bf16(rng.standard_normal((2, H, 128, R)) / math.sqrt(1.65 * R))


def pool_of(kv, P):
    """The positions in pages 1, 3, 5, ... of a pool whose other slots are NaN."""
    need = -(-len(kv) // P)
    pool = np.full((2 * need + 1, P, kv.shape[1]), np.nan)
    table = 1 + 2 * np.arange(need, dtype=np.int32)
    t = np.arange(len(kv))
    pool[table[t // P], t % P] = kv
    return table, pool


def bound_of(q, kv, q_start, w, scale, causal):
    """The fp64 outputs [C, H, 128] and what the kernel's roundings may move them by:
    - the output to bf16, 2^-8 of it;
    - values and weights to fp16, 2^-11 of each; but a value is held beside a power of two for its 128 positions,
      which puts their largest at 2^14 at least, so no better than half of fp16's least step, 2^-39 of that largest;
      and of the products of weight and such a largest value the row's largest is at least 2^23, so a weight below
      fp16's normal range is off by 2^-25 of values below 2^15: 2^-33 of the row's largest product, a position;
    - a value's sum of R products in fp32 (2^-23 an addition, if it cuts off), the exponentials, 2^-19;
    - the scores: the 128 expanded key channels to bf16 (2^-8 of each), sums in fp32, every weight by e^(2 error)."""
    C, H, _ = q.shape
    n, R = len(kv), kv.shape[1] - 64
    ref, bound = np.zeros((C, H, 128)), np.zeros((C, H, 128))
    seen = (np.arange(n) <= q_start + np.arange(C)[:, None]) if causal else np.ones((C, n), bool)
    for h in range(H):
        k, v = O.expand(kv, w[0][h], w[1][h])
        wt = O.softmax(np.where(seen, scale * (q[:, h] @ k.T), -np.inf))
        aq, sums = np.abs(q[:, h]), np.abs(kv[:, :R]) @ np.abs(w[1][h]).T
        off = (aq[:, :128] @ (np.abs(k[:, :128]).T * 2.0 ** -8 + (np.abs(kv[:, :R]) @ np.abs(w[0][h]).T).T * R * 2.0 ** -23)
               + aq @ np.abs(k).T * 192 * 2.0 ** -23)
        err = abs(scale) * np.where(seen, off, 0).max(1)[:, None]
        pad = np.pad(np.abs(v).max(1), (0, -n % 128)).reshape(-1, 128).max(1)
        top = np.repeat(pad, 128)[:n]                  # the largest value of a position's 128
        ref[:, h] = wt @ v
        bound[:, h] = (np.abs(ref[:, h]) * 2.0 ** -8 + wt @ np.abs(v) * (2.0 ** -10 + 2.0 ** -19 + np.expm1(2 * err))
                       + wt @ sums * R * 2.0 ** -23 + (wt @ top)[:, None] * 2.0 ** -39
                       + (n * 2.0 ** -33) * (wt * top).max(1)[:, None])
    return ref, bound


def run(q, kv, q_start, w, scale=T.SCALE, causal=True, P=64, expect=0):
    table, pool = pool_of(kv, P)
    C, H, _ = q.shape
    out = torch.full((C, H, 128), float("nan"), device="cuda").bfloat16()
    ws = jf.latent_prefill_workspace(q_start, C, H)
    jf.jf_latent_prefill_attn(T.gpu_pool(pool), ints(table), gpu(q), q_start, gpu(w[0]), gpu(w[1]), scale, causal, out, ws)
    assert jf.workspace_status(ws) == expect
    return f64(out)


def check(q, kv, q_start, w, scale=T.SCALE, causal=True, P=64, expect=0, norm=0.004):
    """Every element within its bound; and each head's error, of its norm, within `norm`: the output's rounding is
    2^-8 / sqrt(3) = 0.0023 at most if it falls anywhere in its step, values, weights and scores beside it
    (2^-11 twice, and 2^-8 of 192 channels' terms of either sign) less than that again."""
    ref, bound = bound_of(q, kv, q_start, w, scale, causal)
    got = run(q, kv, q_start, w, scale, causal, P, expect)
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:3], got[bad][:3], ref[bad][:3])
    for h in range(q.shape[1] if norm else 0):
        top = np.abs(ref[:, h]).max()
        off, all_ = np.linalg.norm((got - ref)[:, h] / top), np.linalg.norm(ref[:, h] / top)
        assert off <= norm * all_, (h, off / all_)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("power", [-100, -60, -30, -24, -20, -16, -8, 8, 20, 60, 100])
def test_values_of_any_magnitude(power, causal):
    rng = np.random.default_rng(200 + power)
    kv, q, w = T.rows(rng, 200, 256), T.bf16(rng.standard_normal((150, 2, 192))), weights(rng, 2, 256)
    w[1] *= 2.0 ** power
    # values past 65,504 are reported, and come out as any others
    check(q, kv, 50, w, causal=causal, expect=RANGE if power >= 20 else 0)


def test_heads_of_different_magnitudes():
    rng = np.random.default_rng(201)
    kv, q, w = T.rows(rng, 400, 512), T.bf16(rng.standard_normal((130, 6, 192))), weights(rng, 6, 512)
    w[1] *= 2.0 ** np.array([0, -40, 12, -90, -25, 5])[:, None, None]
    check(q, kv, 270, w)


@pytest.mark.parametrize("R,n,C,H", [(256, 700, 700, 2), (512, 5000, 130, 2), (256, 1100, 300, 40)])
@pytest.mark.parametrize("what", ["rise", "fall", "steps", "mixed"])
def test_positions_of_different_magnitudes(R, n, C, H, what):
    """Latents from 2^-100 up along the positions and back, by blocks of 64 and by positions: the first queries see
    the small ones alone, and items of a long history are joined from parts of either kind."""
    rng = np.random.default_rng(202 + n)
    kv, q, w = T.rows(rng, n, R), T.bf16(rng.standard_normal((C, H, 192))), weights(rng, H, R)
    t = np.arange(n)
    power = {"rise": np.floor(100 * t / n) - 100, "fall": -np.floor(100 * t / n), "steps": -60.0 * (t // 64 % 2),
             "mixed": -np.floor(30 * rng.random(n))}[what]
    kv[:, :R] *= 2.0 ** power[:, None]
    check(q, kv, n - C, w, norm=0.004 if what != "rise" else None)


@pytest.mark.parametrize("n,C", [(300, 150), (5000, 100)])
@pytest.mark.parametrize("power,score", [(-12, 8), (-30, 20), (-60, 40), (-110, 30), (-110, 70)])
def test_first_positions_with_most_of_the_weight_and_little_value(n, C, power, score):
    """The sum is theirs, the output the others': weights that are stored as next to nothing still count."""
    rng = np.random.default_rng(203 + n)
    R = 512
    kv, q, w = T.rows(rng, n, R), T.bf16(rng.standard_normal((C, 2, 192))), weights(rng, 2, R)
    kv[:40, :R] *= 2.0 ** power
    kv[:, R] = 0
    kv[:4, R] = T.bf16(np.array([score / 8]))[0]
    q[:, :, 128] = T.bf16(np.array([8 / T.SCALE]))[0]
    check(q, kv, n - C, w, norm=None)


@pytest.mark.parametrize("n,C,zero", [(300, 150, slice(0, 32)), (300, 150, slice(64, 200)), (300, 300, slice(0, 256)),
                                      (5000, 100, slice(100, 4000)), (200, 100, slice(0, 200))])
@pytest.mark.parametrize("power", [0, -50])
def test_latents_of_zero(n, C, zero, power):
    """Positions that hold nothing draw their weight all the same."""
    rng = np.random.default_rng(204 + n)
    R = 256
    kv, q, w = T.rows(rng, n, R), T.bf16(rng.standard_normal((C, 2, 192))), weights(rng, 2, R)
    kv[:, :R] *= 2.0 ** power
    kv[zero, :R] = 0
    kv[zero, R:] *= 2
    check(q, kv, n - C, w, norm=None)


@pytest.mark.parametrize("up", [True, False])
def test_scores_and_magnitudes_against_each_other(up):
    """Scores from -600 to 600 in base e while the values go the other way, 2^-100 to 1."""
    rng = np.random.default_rng(205)
    n, C, R = 900, 150, 512
    kv, q, w = T.rows(rng, n, R), T.bf16(rng.standard_normal((C, 2, 192))), weights(rng, 2, R)
    ramp = np.linspace(-600, 600, n) * (1 if up else -1)
    kv[:, R] = T.bf16(ramp / 8)
    kv[:, :R] *= (2.0 ** (np.floor(-ramp / 12) - 50))[:, None]
    q[:, :, 128] = T.bf16(np.array([8 / T.SCALE]))[0]
    check(q, kv, n - C, w, norm=None)


def test_a_value_that_is_not_finite_beside_small_ones():
    rng = np.random.default_rng(206)
    n, q_start, at, R = 300, 100, 230, 512
    kv, q, w = T.rows(rng, n, R), T.bf16(rng.standard_normal((200, 3, 192))), weights(rng, 3, R)
    kv[:, :R] *= 2.0 ** -40
    clean = run(q, kv, q_start, w)
    ref, bound = bound_of(q, kv, q_start, w, T.SCALE, True)
    kv[at, 17] = np.inf
    got = run(q, kv, q_start, w)
    assert np.isnan(got[at - q_start:]).all()
    assert (np.abs(got - ref) <= bound)[:at - q_start].all() and np.array_equal(got[:130], clean[:130])
