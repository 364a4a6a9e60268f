"""Seeded inputs of the latent cache's tests, and bounds for their outputs."""
import math

import numpy as np
import torch

import paper_2609_17475_gb300 as jf

ROT = 64
SCALE = float(np.float32(1 / math.sqrt(192)))


def bf16(x):
    """bf16-representable fp64 values."""
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().double().numpy()


def gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().cuda()


def f64(t):
    return t.double().cpu().numpy()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def rows(rng, n, R):
    return bf16(rng.standard_normal((n, R + ROT)) * np.concatenate([np.exp(0.5 * rng.standard_normal(R)), np.ones(ROT)]))


def queries(rng, n, H, R):
    q = rng.standard_normal((n, H, R + ROT))
    q[..., :R] *= math.sqrt(128 / (1.65 * R))
    return bf16(q)


def tables(rng, need, spare=2, width=None):
    """Page tables (-1 past a request's pages) over a shuffled pool, and its pages."""
    total = sum(need) + spare
    perm = rng.permutation(total).astype(np.int32)
    t = np.full((len(need), max(max(need), 1) if width is None else width), -1, dtype=np.int32)
    off = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[off:off + n]
        off += n
    return t, total


def filled(rng, R, P, lens, extra=0):
    """fp64 pool [pages, P, R + 64] with lens[b] rows of each request; every other slot is NaN."""
    table, pages = tables(rng, [-(-n // P) + extra for n in lens])
    pool = np.full((pages, P, R + ROT), np.nan)
    for b, n in enumerate(lens):
        t = np.arange(n)
        pool[table[b, t // P], t % P] = rows(rng, n, R)
    return table, pool


def gpu_pool(pool):
    pages, P, d = pool.shape
    return jf.KVPool(gpu(pool).view(torch.uint8).view(pages, P * d * 2), P, 1, d, format=jf.JF_FMT_LATENT16)


def score_error(q, kv, scale, width):
    """What fp32 sums of `width` products may move a score by: 2^-23 of the terms' magnitudes an addition (a sum that
    cuts off instead of rounding)."""
    if len(kv) == 0:
        return 0.0
    return abs(scale) * (np.abs(q) @ np.abs(kv).T).max() * width * 2.0 ** -23


def decode_bound(ref, mass, score):
    """|out - ref|: half a bf16 step of the result (2^-8), the weights' roundings to bf16 over a sum that is off by as
    much (2 x 2^-8 of sum |w c|), the exponentials (2^-20), and scores off by `score`: every weight by e^(2 score)."""
    return np.abs(ref) * 2.0 ** -8 + mass * (2.0 ** -7 + 2.0 ** -19 + math.expm1(2 * score)) + 2.0 ** -130
