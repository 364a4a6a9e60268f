"""Eviction by accumulated weight on the GPU: kept positions, weights and the compacted pages, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import kv8 as O
from tests import kv8_cases as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def evict(L, pool, table, ctx, w, budget, sinks, recent, dst, with_weights=True):
    g = C.gpu_pool(L, pool.copy())
    B = len(ctx)
    kept = torch.full((B, L.Hkv, budget), -7, dtype=torch.int32, device=DEV)
    wout = torch.full((B, L.Hkv, budget), -7.0, device=DEV) if with_weights else None
    n, err = torch.full((B,), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    jf.jf_kv8_evict(g, C.ints(table), C.ints(ctx), torch.from_numpy(w).to(DEV), budget, sinks, recent, C.ints(dst), n,
                    wout, kept, err)
    return g, kept, wout, n, int(err)


def check(hkv, d, p, ctx, budget, sinks, recent, make, seed=0, spread=6):
    rng = np.random.default_rng(seed + sum(ctx) + budget)
    extra = [-(-min(n, budget) // p) for n in ctx]
    L, table, pool = C.filled(rng, hkv, p, d, ctx, fill=0xFF, spread=spread, extra=extra)
    own = [-(-n // p) for n in ctx]
    dst = np.full((len(ctx), max(max(extra), 1)), -1, dtype=np.int32)
    src = np.full((len(ctx), max(max(own), 1)), -1, dtype=np.int32)
    for b in range(len(ctx)):
        src[b, :own[b]] = table[b, :own[b]]
        dst[b, :extra[b]] = table[b, own[b]:own[b] + extra[b]]
    w = make(rng, (len(ctx), hkv, max(max(ctx), 1) + 5)).astype(np.float32)
    g, kept, wout, n, err = evict(L, pool, src, ctx, w, budget, sinks, recent, dst)
    want_kept, want_w = O.evict(pool, L, src, ctx, w, budget, sinks, recent, dst)
    assert err == 0
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(wout.cpu().numpy().view(np.int32), want_w.view(np.int32))
    assert n.tolist() == [min(c, budget) for c in ctx]
    assert np.array_equal(g.data.cpu().numpy(), pool)       # the compacted pages, and nothing else


def uneven(rng, shape):
    return np.exp(2 * rng.standard_normal(shape)) * (rng.random(shape) < 0.7)


def ties(rng, shape):
    return rng.integers(0, 4, shape) / 4


def odd(rng, shape):
    """NaN, infinities, signed zeros, negative and subnormal weights."""
    pick = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.5, 1e-40, -1e-40, 2.0, 3e38])
    return pick[rng.integers(0, len(pick), shape)]


@pytest.mark.parametrize("make", [uneven, ties, odd])
@pytest.mark.parametrize("hkv,d,p,ctx,budget,sinks,recent", [
    (2, 128, 64, [300], 100, 4, 32),
    (1, 256, 128, [1, 0, 33, 500, 129], 33, 0, 0),
    (3, 128, 256, [700, 64], 64, 0, 64),
    (4, 256, 64, [65], 64, 1, 0),
    (1, 128, 128, [2000, 31], 1, 0, 0),
    (2, 128, 64, [1025, 1024], 1024, 1000, 24),
])
def test_evict(make, hkv, d, p, ctx, budget, sinks, recent):
    check(hkv, d, p, ctx, budget, sinks, recent, make)


def test_evict_long_rows():
    """Rows of tens of thousands of positions (odd lengths), keys that share long prefixes."""
    check(1, 128, 256, [40003, 16385], 5001, 4, 77, lambda r, s: 1 + r.integers(0, 1 << 12, s) * 2.0 ** -23, spread=0)


@pytest.mark.parametrize("skew", [0, 1, 2, 3])
@pytest.mark.parametrize("n", [101, 130, 4097, 20001])
def test_evict_weights_at_any_address(skew, n):
    """Rows of weights that begin and end off a 16-byte boundary, in every way; nothing beside them is read as theirs."""
    hkv, d, p, budget = 2, 128, 64, 100
    rng = np.random.default_rng(40 * n + skew)
    own, extra = -(-n // p), -(-budget // p)
    L, table, pool = C.filled(rng, hkv, p, d, [n], extra=[extra])
    src, dst = table[:, :own].copy(), table[:, own:own + extra].copy()
    w = uneven(rng, (1, hkv, n)).astype(np.float32)      # row 1 begins n weights after row 0
    wide = torch.full((hkv * n + 8,), 1e30, device=DEV)
    wide[skew:skew + hkv * n] = torch.from_numpy(w.reshape(-1)).to(DEV)
    view = wide[skew:skew + hkv * n].view(1, hkv, n)
    g = C.gpu_pool(L, pool.copy())
    kept, wout = torch.empty(1, hkv, budget, dtype=torch.int32, device=DEV), torch.empty(1, hkv, budget, device=DEV)
    m, err = torch.empty(1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    jf.jf_kv8_evict(g, C.ints(src), C.ints([n]), view, budget, 3, 8, C.ints(dst), m, wout, kept, err)
    want_kept, want_w = O.evict(pool, L, src, [n], w, budget, 3, 8, dst)
    assert int(err) == 0 and int(m) == budget
    assert np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(wout.cpu().numpy(), want_w)
    assert np.array_equal(g.data.cpu().numpy(), pool)


def test_evict_codes_of_nan():
    """Codes that are NaN (of either sign) stay NaN, in the one code it has, and scale nothing."""
    hkv, d, p, n, budget = 2, 128, 64, 150, 70
    rng = np.random.default_rng(77)
    L, table, pool = C.filled(rng, hkv, p, d, [n], extra=[2], spread=3)
    src, dst = table[:, :3].copy(), table[:, 3:5].copy()
    for t in range(0, n, 7):                             # byte t of each position's row, K and V
        page, slot = pool[table[0, t // p]], t % p
        for side in range(2):
            for h in range(hkv):
                at = (side * hkv + h) * p * d + slot * d + t % d
                page[at] = (0xFF, 0x7F)[t % 2]
    w = uneven(rng, (1, hkv, n)).astype(np.float32)
    g, kept, wout, m, err = evict(L, pool, src, [n], w, budget, 0, 9, dst)
    want_kept, _ = O.evict(pool, L, src, [n], w, budget, 0, 9, dst)
    assert err == 0 and np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(g.data.cpu().numpy(), pool)


@pytest.mark.parametrize("make", [uneven, ties, odd])
def test_evict_rows_too_long_for_shared_memory(make):
    """Rows of weights past what a cluster's shared memory holds, whatever the contexts: short contexts in them, pages
    and all, and one context of the whole row (its pages repeat) by its kept positions and weights."""
    rng = np.random.default_rng(50)
    hkv, d, p, budget, stride = 1, 128, 64, 300, 800_003
    ctx = [9001, 300, 301, 0]
    own, extra = [-(-n // p) for n in ctx], [-(-min(n, budget) // p) for n in ctx]
    L, table, pool = C.filled(rng, hkv, p, d, ctx, extra=extra)
    src, dst = np.full((4, max(own)), -1, np.int32), np.full((4, max(extra)), -1, np.int32)
    for b in range(4):
        src[b, :own[b]], dst[b, :extra[b]] = table[b, :own[b]], table[b, own[b]:own[b] + extra[b]]
    w = np.zeros((4, hkv, stride), np.float32)
    w[:, :, :9001] = make(rng, (4, hkv, 9001))
    g, kept, wout, n, err = evict(L, pool, src, ctx, w, budget, 4, 32, dst)
    want_kept, want_w = O.evict(pool, L, src, ctx, w, budget, 4, 32, dst)
    assert err == 0 and np.array_equal(kept.cpu().numpy(), want_kept)
    assert np.array_equal(wout.cpu().numpy().view(np.int32), want_w.view(np.int32))
    assert np.array_equal(g.data.cpu().numpy(), pool)

    n, budget = stride - 2, 5003
    w = make(rng, (1, hkv, stride)).astype(np.float32)
    src = np.zeros((1, -(-n // p)), np.int32) + table[0, 0]
    dst = np.setdiff1d(np.arange(len(pool)), table[0, :1])[None, :-(-budget // p)].astype(np.int32)
    _, kept, wout, m, err = evict(L, pool, src, [n], w, budget, 4, 32, dst)
    at = O.keep(w[0, 0, :n], budget, 4, 32)
    assert err == 0 and int(m) == budget and np.array_equal(kept[0, 0].cpu().numpy(), at)
    assert np.array_equal(wout[0, 0].cpu().numpy().view(np.int32), w[0, 0, at].view(np.int32))


def test_evict_then_decode_sees_the_kept_positions():
    rng = np.random.default_rng(5)
    L, table, pool = C.filled(rng, 2, 64, 128, [500, 90], extra=[2, 2])
    src, dst = table[:, :8].copy(), np.stack([table[0, 8:10], table[1, 2:4]])
    w = uneven(rng, (2, 2, 500)).astype(np.float32)
    g, kept, _, n, err = evict(L, pool, src, [500, 90], w, 100, 4, 16, dst, with_weights=False)
    assert err == 0 and n.tolist() == [100, 90]
    q = torch.randn(2, 8, 128, device=DEV).bfloat16()
    out, ws = torch.empty_like(q), jf.decode_workspace(2, 8, 2, 128, 3)
    jf.jf_paged_decode_attn(g, C.ints(dst), n, q, 0.1, out, ws, 3)
    assert jf.workspace_status(ws) == 0
    after = g.data.cpu().numpy()
    for b in range(2):
        k, v = O.read(after, L, dst[b], int(n[b]))
        ref, p, mass = O.attend(k, v, q[b:b + 1].double().cpu().numpy(), float(np.float32(0.1)))
        e = np.abs(out[b].double().cpu().numpy() - ref[0])
        assert (e <= C.out_bound(ref[0], mass[0], 100, np.abs(v).max())).all()


def test_evict_reports_and_refuses():
    rng = np.random.default_rng(6)
    L, table, pool = C.filled(rng, 1, 64, 128, [200, 130])
    w = uneven(rng, (2, 1, 200)).astype(np.float32)
    P, G = jf.binding.JF_DEV_ERR_POSITION, jf.binding.JF_DEV_ERR_PAGE_ID
    spare = sorted(set(range(len(pool))) - set(table[0, :4]) - set(table[1, :3]))
    dst = np.array([[spare[0]], [spare[1]]], dtype=np.int32)
    # a context past its weights or its table: kept as empty, the other request done
    for ctx in ([201, 130], [-1, 130], [64 * 4 + 1, 130]):
        g, kept, _, n, err = evict(L, pool, table, ctx, w, 40, 2, 2, dst)
        assert err == P and n.tolist() == [0, 40] and (kept[0] == -1).all()
        want = pool.copy()
        wk, _ = O.evict(want, L, table[1:], [130], w[1:], 40, 2, 2, dst[1:])
        assert np.array_equal(kept[1:].cpu().numpy(), wk) and np.array_equal(g.data.cpu().numpy(), want)
    # a source page outside the pool reads as zeros; a destination one is not written
    bad = table.copy()
    bad[0, 0] = -1
    assert evict(L, pool, bad, [200, 130], w, 40, 2, 2, dst)[4] == G
    assert evict(L, pool, table, [200, 130], w, 40, 2, 2, np.array([[-1], [spare[1]]]))[4] == G
    # a destination row too short for the budget
    assert evict(L, pool, table, [200, 130], w, 65, 2, 2, dst)[4] == P
    for budget, sinks, recent in ((0, 0, 0), (4, 3, 2), (4, -1, 0), (4, 0, -1)):
        with pytest.raises((jf.JfError, RuntimeError)) as e:
            evict(L, pool, table, [200, 130], w, budget, sinks, recent, dst)
        assert isinstance(e.value, jf.JfError) and e.value.status == jf.binding.JF_ERR_INVALID_ARG
