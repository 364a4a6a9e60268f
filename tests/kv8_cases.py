"""Seeded inputs of the 8-bit cache's tests, and pools built by the oracle."""
import numpy as np
import torch

import paper_2609_17475_gb300 as jf
from oracle import kv8 as O


def rows(rng, n, hkv, d, spread=0):
    """bf16-representable fp64 rows [n, Hkv, D]; `spread`: each block of 32 rows times 2^[-spread, spread]."""
    x = rng.standard_normal((n, hkv, d))
    x[:, :, rng.integers(0, d, 4)] *= 20
    if spread:
        e = rng.integers(-spread, spread + 1, (-(-n // 32), hkv, 1))
        x *= np.exp2(np.repeat(e, 32, 0)[:n])
    return torch.from_numpy(x).bfloat16().double().numpy()


def bf16(x, device="cuda"):
    return torch.from_numpy(np.ascontiguousarray(x)).bfloat16().to(device)


def tables(rng, need, spare=2):
    """Page tables (-1 past a request's pages) over a shuffled pool, and its pages."""
    total = sum(need) + spare
    perm = rng.permutation(total).astype(np.int32)
    t = np.full((len(need), max(max(need), 1)), -1, dtype=np.int32)
    off = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[off:off + n]
        off += n
    return t, total


def filled(rng, hkv, p, d, ctx, fill=0xFF, spread=0, extra=None):
    """An oracle pool that holds ctx[b] rows of each request; other bytes are `fill` (0xff: NaN codes and
    NaN scales).  extra[b]: further pages of request b's table."""
    L = O.Layout(hkv, p, d)
    need = [-(-n // p) + (extra[b] if extra else 0) for b, n in enumerate(ctx)]
    table, pages = tables(rng, need)
    pool = O.new_pool(L, pages, fill)
    off = np.concatenate([[0], np.cumsum(ctx)]).astype(np.int64)
    k, v = rows(rng, int(off[-1]), hkv, d, spread), rows(rng, int(off[-1]), hkv, d, spread)
    O.append(pool, L, table, [0] * len(ctx), off, k, v)
    return L, table, pool


def gpu_pool(L, pool):
    return jf.KVPool(torch.from_numpy(pool).cuda(), L.P, L.Hkv, L.D, format=jf.JF_FMT_E4M3_B32)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def out_bound(ref, mass, n, top):
    """What |out - ref| may be: half a bf16 step of the result (2^-8 of it, and 2^-133 for subnormal ones),
    the weights' rounding to fp16 (2^-11) and the exponential's error, together below 2^-10 of sum |w v|, and
    fp16's floor: a weight times scale below 2^-34 of the largest one, `top`, loses up to 2^-34 * 448 of it for
    each of the n positions."""
    return np.abs(ref) * 2.0 ** -8 + mass * 2.0 ** -10 + n * top * 448 * 2.0 ** -34 + 2.0 ** -130
