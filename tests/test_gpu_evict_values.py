"""Eviction of rows whose values or pages are out of the ordinary, bit for bit against the oracle."""
import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import kv8 as O
from tests import kv8_cases as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def evict(L, pool, src, n, w, budget, dst):
    """The GPU's pool, kept positions, weights, lengths and error flag; nothing protected."""
    g, B = C.gpu_pool(L, pool.copy()), len(n)
    kept = torch.full((B, L.Hkv, budget), -7, dtype=torch.int32, device=DEV)
    wout, m, err = torch.full((B, L.Hkv, budget), -7.0, device=DEV), C.ints([-7] * B), C.ints([0])
    jf.jf_kv8_evict(g, C.ints(src), C.ints(n), torch.from_numpy(w).to(DEV), budget, 0, 0, C.ints(dst), m, wout, kept, err)
    return g.data.cpu().numpy(), kept.cpu().numpy(), wout.cpu().numpy(), m.tolist(), int(err)


def same(got, want, L, pages):
    """Codes and scales of the given pages, apart from anything else."""
    for a, b in zip(L.views(got[pages]), L.views(want[pages])):
        assert np.array_equal(a.view(np.uint8), b.view(np.uint8))


@pytest.mark.parametrize("zero", ["k", "v", "both"])
@pytest.mark.parametrize("scale", [0, -30, 34])          # of the ordinary rows: a power of two
@pytest.mark.parametrize("d,p,budget", [(128, 64, 33), (128, 64, 32), (256, 128, 65), (256, 64, 97)])
def test_zero_rows_stay_zero(zero, scale, d, p, budget):
    """Rows of zeros, of either sign, kept from blocks that also hold ordinary rows: as a whole block of the
    destination, as a last block of one row, and beside rows of a scale far below their own block's."""
    hkv, n = 2, 300
    rng = np.random.default_rng(budget + d + scale)
    L = O.Layout(hkv, p, d)
    need = [-(-n // p), -(-budget // p)]
    table, pages = C.tables(rng, need)
    src, dst = table[:1, :need[0]].copy(), table[1:, :need[1]].copy()
    k, v = C.rows(rng, n, hkv, d) * 2.0 ** scale, C.rows(rng, n, hkv, d) * 2.0 ** scale
    small = np.arange(n) >= 256                           # two blocks whose rows are far smaller
    k[small] *= 2.0 ** -40
    v[small] *= 2.0 ** -40
    none = (np.arange(n) % 5 == 2) & ~small               # a few rows of zeros in every ordinary block
    for name, x in (("k", k), ("v", v)):
        if zero in (name, "both"):
            x[none] = 0.0
            x[none, :, ::3] = -0.0
    pool = O.new_pool(L, pages, 0xFF)
    O.append(pool, L, src, [0], np.array([0, n]), k, v)
    # the zero rows are kept first; what the budget has left goes to the small rows
    w = np.where(none, 2.0, np.where(small, 1.0, 0.0)).astype(np.float32)
    w = np.ascontiguousarray(np.broadcast_to(w, (1, hkv, n)))
    got, kept, wout, m, err = evict(L, pool, src, [n], w, budget, dst)
    want_kept, want_w = O.evict(pool, L, src, [n], w, budget, 0, 0, dst)
    assert err == 0 and m == [budget] and np.array_equal(kept, want_kept) and np.array_equal(wout, want_w)
    same(got, pool, L, dst[0])
    assert np.array_equal(got, pool)
    for x, name in zip(O.read(got, L, dst[0], budget), "kv"):
        assert np.isfinite(x).all()
        if zero in (name, "both"):
            assert not x[np.isin(want_kept[0, 0], np.flatnonzero(none))].any()


def test_pages_outside_the_pool_by_their_outputs():
    """A source page outside the pool gives rows of zeros, a destination one and a destination row too short are not
    written; kept positions, weights and all other bytes are those of the definition."""
    rng = np.random.default_rng(6)
    hkv, d, p, n, budget = 2, 128, 64, [200, 130], 70
    L, table, pool = C.filled(rng, hkv, p, d, n, extra=[2, 2])
    src = np.stack([table[0, :4], np.append(table[1, :3], -1)])
    dst = np.stack([table[0, 4:6], table[1, 3:5]])
    w = rng.random((2, hkv, 200), dtype=np.float32)
    page_bit, pos_bit = jf.binding.JF_DEV_ERR_PAGE_ID, jf.binding.JF_DEV_ERR_POSITION

    # request 0's second page lies outside: as if its rows had been zeros
    for outside in (-1, len(pool), 1 << 30):
        bad = src.copy()
        bad[0, 1] = outside
        got, kept, wout, m, err = evict(L, pool, bad, n, w, budget, dst)
        clean = pool.copy()
        clean[src[0, 1]] = 0
        at = 2 * hkv * p * d
        clean[src[0, 1], at:] = np.full(2 * hkv * (p // 32), 2.0 ** -40, np.float32).view(np.uint8)
        want_kept, want_w = O.evict(clean, L, src, n, w, budget, 0, 0, dst)
        want = pool.copy()
        want[dst.reshape(-1)] = clean[dst.reshape(-1)]
        assert err == page_bit and m == [budget, budget]
        assert np.array_equal(kept, want_kept) and np.array_equal(wout, want_w) and np.array_equal(got, want)

    # request 0's destination: its second page outside, or not there
    want = pool.copy()
    want_kept, want_w = O.evict(want, L, src, n, w, budget, 0, 0, dst)
    want[dst[0, 1]] = pool[dst[0, 1]]
    for outside in (-1, len(pool)):
        bad = dst.copy()
        bad[0, 1] = outside
        got, kept, wout, m, err = evict(L, pool, src, n, w, budget, bad)
        assert err == page_bit and m == [budget, budget]
        assert np.array_equal(kept, want_kept) and np.array_equal(wout, want_w) and np.array_equal(got, want)
    want[dst[1, 1]] = pool[dst[1, 1]]
    got, kept, wout, m, err = evict(L, pool, src, n, w, budget, dst[:, :1].copy())
    assert err == pos_bit and m == [budget, budget]
    assert np.array_equal(kept, want_kept) and np.array_equal(wout, want_w) and np.array_equal(got, want)
