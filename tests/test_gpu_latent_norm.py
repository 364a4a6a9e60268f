"""Latent decode on the GPU by the norm of its error: long contexts, in which one tile more or less is lost in what an
element's bound allows for, and large scores, where the worst case of their sums says little."""
import numpy as np
import pytest

from oracle import latent as O
from tests import latent_cases as T
from tests import test_gpu_latent as G
from tests.latent_cases import f64

pytestmark = pytest.mark.gpu

# The output and the weights are rounded to bf16: 2^-8 / sqrt(3) of each at most if a rounding falls anywhere in its
# step.  The weights' are as many as there are positions, of either sign, as are the terms of the output itself, so
# that they move it by the same part: together sqrt(2) 2^-8 / sqrt(3).  Scores are off by 2^-24 of sums of 576 terms.
# (Few positions do not average: 64 of them, a few with most of the weight, may all be rounded one way, by 2^-8 each.
# Below 256 the elements' bound holds alone.)
LIMIT = 0.0032


def off_by(got, ref):
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


def check(out, q, kv):
    """Every head's error within LIMIT of its norm; and the oracle without one tile of 128 positions is not: the bound
    would tell."""
    if len(kv) < 256:
        G.check(out, q, kv, T.SCALE)
        return
    ref = O.decode(q, kv, T.SCALE)[0]
    got = f64(out)
    for h in range(len(q)):
        assert off_by(got[h], ref[h]) <= LIMIT, (h, off_by(got[h], ref[h]))
    n, h = len(kv), len(q) // 2
    for at in (0, n // 256 * 128, n // 128 * 128 - 128):
        less = O.decode(q[h:h + 1], np.delete(kv, np.s_[at:at + 128], 0), T.SCALE)[0]
        assert off_by(less, ref[h:h + 1]) > LIMIT, at


@pytest.mark.parametrize("R,H,P,ctx", [(512, 16, 64, [20000]), (512, 128, 128, [20000]), (256, 20, 256, [9000, 5000]),
                                       (512, 130, 64, [9001]), (512, 3, 128, [40000]), (256, 128, 64, [17000, 64, 12345])])
def test_long_decodes(R, H, P, ctx):
    rng = np.random.default_rng(300 + R + H)
    table, pool = T.filled(rng, R, P, ctx)
    q = T.queries(rng, len(ctx), H, R)
    out, st = G.run_decode(table, pool, ctx, q, T.SCALE)
    assert st == 0
    for b, n in enumerate(ctx):
        check(out[b], q[b], O.gather(pool, table[b], n))


@pytest.mark.parametrize("R,H,P,sizes,plens,ctx", [
    (512, 128, 64, [2, 3], [9000, 4001], [1, 500, 0, 2000, 300]),
    (512, 16, 128, [20, 9], [20000, 6001], [37 * i for i in range(29)]),
    (256, 200, 64, [2, 1], [12000, 64], [10, 0, 7000]),
])
def test_long_prefixes(R, H, P, sizes, plens, ctx):
    rng = np.random.default_rng(301 + R + H)
    both, pool = T.filled(rng, R, P, plens + ctx)
    off = np.concatenate([[0], np.cumsum(sizes)]).tolist()
    q = T.queries(rng, len(ctx), H, R)
    out, st = G.run_prefix(pool, both[:len(plens)], plens, off, both[len(plens):], ctx, q, T.SCALE)
    assert st == 0
    for g, n in enumerate(plens):
        for b in range(off[g], off[g + 1]):
            kv = np.concatenate([O.gather(pool, both[g], n), O.gather(pool, both[len(plens) + b], ctx[b])])
            check(out[b], q[b], kv)


@pytest.mark.parametrize("R,scale", [(512, 30.0), (256, 30.0), (512, -7.0), (512, 1.0)])
def test_large_scores_of_exact_sums(R, scale):
    """Queries and keys in eighths up to 1: their sums are exact in fp32, so a score is off by its scaling alone,
    2^-23 of it, and a weight by e to the power of twice that."""
    rng = np.random.default_rng(302 + R)
    n, H = 3000, 16
    kv, q = rng.integers(-8, 9, (n, R + 64)) / 8, rng.integers(-8, 9, (1, H, R + 64)) / 8
    table, pool = T.filled(rng, R, 64, [n])
    t = np.arange(n)
    pool[table[0, t // 64], t % 64] = kv
    out, st = G.run_decode(table, pool, [n], q, scale)
    assert st == 0
    ref, mass = O.decode(q[0], kv, scale)
    score = abs(scale) * np.abs(q[0] @ kv.T).max() * 2.0 ** -23
    got = f64(out[0])
    # a weight below fp32's least normal number, 2^-126 of the largest, may count as none: of latents up to 1 each
    bad = ~(np.abs(got - ref) <= T.decode_bound(ref, mass, score) + n * 2.0 ** -126)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:5], got[bad][:5], ref[bad][:5])
    assert score < 0.002 and off_by(got, ref) <= LIMIT + 2 * score
