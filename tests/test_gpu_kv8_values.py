"""Attention over the 8-bit cache for values out of the ordinary: elements that are no numbers, scores that are all
zero, queries whose elements differ by many powers of two."""
import math

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import kv8 as O
from tests import kv8_cases as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def prefill(L, table, pool, start, q, scale, splits=1, causal=True):
    """The output [C, Hq, D] of one request's chunk q, through the chunk call or in `splits` history ranges."""
    g, out = C.gpu_pool(L, pool), torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    if splits == 1:
        ws = jf.prefill_chunk_workspace(g, start, q.shape[0], q.shape[1])
        jf.jf_prefill_chunk_attn(g, C.ints(table)[0], C.bf16(q), start, scale, causal, out, ws)
    else:
        ws = jf.prefill_batch_workspace(q.shape[0], q.shape[1], L.D, splits, format=jf.JF_FMT_E4M3_B32)
        ws[256:] = 0xFF
        jf.jf_prefill_batch_attn(g, C.ints(table), [start], [q.shape[0]], C.bf16(q), scale, causal, out, ws, splits)
    assert jf.workspace_status(ws) == 0
    return out.double().cpu().numpy()


def decode(L, table, pool, ctx, q, scale, splits, weigh=False):
    g, B = C.gpu_pool(L, pool), len(ctx)
    out, w = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV), None
    if weigh:
        w = torch.zeros(B, L.Hkv, max(ctx), device=DEV)
        ws = jf.decode_weights_workspace(B, q.shape[1], L.Hkv, L.D, splits, max(ctx))
        ws[256:] = 0
        jf.jf_paged_decode_weights_attn(g, C.ints(table), C.ints(ctx), C.bf16(q), scale, out, None, w, ws, splits)
        w = w.double().cpu().numpy()
    else:
        ws = jf.decode_workspace(B, q.shape[1], L.Hkv, L.D, splits)
        jf.jf_paged_decode_attn(g, C.ints(table), C.ints(ctx), C.bf16(q), scale, out, ws, splits)
    assert jf.workspace_status(ws) == 0
    return out.double().cpu().numpy(), w


def queries(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape)).bfloat16().double().numpy()


# --------------------------------------------------------------------------
# elements that are no numbers
# --------------------------------------------------------------------------
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("hq,hkv,d,start,splits", [(4, 2, 128, 200, 1), (6, 1, 256, 500, 1), (4, 2, 128, 300, 3),
                                                   (6, 1, 256, 300, 4)])
def test_prefill_of_a_query_that_is_no_number(bad, hq, hkv, d, start, splits):
    """A query row with an infinity or a NaN has no softmax: its output is NaN throughout, whatever the split; the
    other rows' outputs are those of the chunk without it."""
    rng = np.random.default_rng(d + splits)
    c = 40
    L, table, pool = C.filled(rng, hkv, 64, d, [start + c])
    q = queries(rng, c, hq, d)
    want = prefill(L, table, pool, start, q, 0.1, splits)
    assert np.isfinite(want).all()
    rows = [(0, 0, 0), (7, hq - 1, d - 1), (39, 1, 17)]
    hit = np.zeros((c, hq), dtype=bool)
    for i, h, j in rows:
        q[i, h, j] = bad
        hit[i, h] = True
    got = prefill(L, table, pool, start, q, 0.1, splits)
    assert np.isnan(got[hit]).all()
    assert np.array_equal(got[~hit], want[~hit])


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_prefill_of_a_query_that_is_no_number_in_a_divided_wave(bad):
    """The same where a chunk's last pairs have their histories in parts (80 pairs: 4 left over)."""
    rng = np.random.default_rng(5)
    hq, hkv, d, p, start, c = 24, 4, 256, 256, 3400, 840
    pages = -(-(start + c) // p)
    g = jf.KVPool.allocate(pages, p, hkv, d, format=jf.JF_FMT_E4M3_B32)
    table = C.ints(rng.permutation(pages)[None])
    torch.manual_seed(1)
    x = [torch.randn(start + c, hkv, d, device=DEV).bfloat16() for _ in range(2)]
    jf.jf_kv8_append(g, table, C.ints([0]), C.ints([0, start + c]), *x)
    q = torch.randn(c, hq, d, device=DEV).bfloat16()
    ws = jf.prefill_chunk_workspace(g, start, c, hq)
    assert ws.numel() > 256
    outs = []
    hit = torch.zeros(c, hq, dtype=torch.bool, device=DEV)
    for i in (0, 3, 400, 839):       # the parts hold the first rows of the chunk
        hit[i, i % hq] = True
    for poison in (False, True):
        if poison:
            for i, h in hit.nonzero().tolist():
                q[i, h, 5] = bad
        out = torch.full_like(q, 7.0)
        jf.jf_prefill_chunk_attn(g, table[0], q, start, 1 / 16, True, out, ws)
        assert jf.workspace_status(ws) == 0
        outs.append(out)
    assert torch.isnan(outs[1][hit]).all() and torch.equal(outs[1][~hit], outs[0][~hit])


@pytest.mark.parametrize("splits", [1, 3])
def test_prefill_of_keys_that_are_no_numbers(splits):
    """Keys that are NaN reach every query that sees one, and no other, also where a whole range of them is."""
    rng = np.random.default_rng(6)
    hq, hkv, d, start, c = 4, 2, 128, 250, 40
    L, table, pool = C.filled(rng, hkv, 64, d, [start + c])
    q = queries(rng, c, hq, d)
    want = prefill(L, table, pool, start, q, 0.1, splits)
    for t0, t1 in ((270, 271), (0, 290)):                  # one key; all of them
        p = pool.copy()
        codes, _ = L.views(p)
        for t in range(t0, t1):
            p[table[0, t // 64], (t % 64) * d + 3] = 0x7F      # KV head 0's key
        got = prefill(L, table, p, start, q, 0.1, splits)
        sees = start + np.arange(c) >= t0
        assert np.isnan(got[sees][:, :2]).all()
        assert np.array_equal(got[:, 2:], want[:, 2:]) and np.array_equal(got[~sees], want[~sees])


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("hq,hkv,d,ctx,splits", [(4, 2, 128, [200, 1, 17], 1), (6, 1, 256, [5000, 64, 3], 9)])
def test_decode_of_a_query_that_is_no_number(weigh, bad, hq, hkv, d, ctx, splits):
    """A head with an infinity or a NaN has no softmax: its output and its KV head's weights are NaN; the other heads'
    are those of the call without it."""
    rng = np.random.default_rng(d)
    L, table, pool = C.filled(rng, hkv, 64, d, ctx)
    q = queries(rng, len(ctx), hq, d)
    want, w0 = decode(L, table, pool, ctx, q, 0.1, splits, weigh)
    hit = np.zeros((len(ctx), hq), dtype=bool)
    for b, h, j in ((0, hq - 1, 5), (1, 0, d - 1), (2, 1, 0)):
        q[b, h, j] = bad
        hit[b, h] = True
    got, w = decode(L, table, pool, ctx, q, 0.1, splits, weigh)
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], want[~hit])
    if weigh:
        kv = hit.reshape(len(ctx), hkv, -1).any(-1)
        for b, n in enumerate(ctx):
            assert np.isnan(w[b, kv[b], :n]).all() and np.array_equal(w[b, ~kv[b], :n], w0[b, ~kv[b], :n])


@pytest.mark.parametrize("ctx,bad", [(1, [0]), (40, range(40)), (3000, [2999]), (3000, range(3000)),
                                     (3000, range(512, 1024))])
@pytest.mark.parametrize("splits", [1, 8])
def test_decode_of_keys_that_are_no_numbers(ctx, bad, splits):
    """Keys that are NaN make their KV head's outputs NaN, however many of them a warp or a piece holds."""
    rng = np.random.default_rng(ctx)
    hq, hkv, d = 4, 2, 128
    L, table, pool = C.filled(rng, hkv, 64, d, [ctx])
    q = queries(rng, 1, hq, d)
    want, _ = decode(L, table, pool, [ctx], q, 0.1, splits)
    for t in bad:
        pool[table[0, t // 64], (t % 64) * d + 3] = 0x7F       # KV head 0's key
    got, _ = decode(L, table, pool, [ctx], q, 0.1, splits)
    assert np.isnan(got[0, :2]).all() and np.array_equal(got[0, 2:], want[0, 2:])


# --------------------------------------------------------------------------
# scores that are all zero
# --------------------------------------------------------------------------
@pytest.mark.parametrize("scale", [2.0 ** -12, 2.0 ** -40, 0.0, 1 / 16])
@pytest.mark.parametrize("splits", [1, 2])
def test_prefill_of_zero_queries_over_zero_keys(scale, splits):
    """Queries of zeros, keys of zeros (whose blocks have the smallest scale), a small softmax scale: each query's
    output is the mean of the values it sees, and those it does not see stay out."""
    rng = np.random.default_rng(7)
    hq, hkv, d, start, c = 2, 1, 128, 70, 50
    n = start + c
    L = O.Layout(hkv, 64, d)
    table, pages = C.tables(rng, [2])
    pool = O.new_pool(L, pages, 0xFF)
    v = C.rows(rng, n, hkv, d)
    O.append(pool, L, table, [0], np.array([0, n]), np.zeros((n, hkv, d)), v)
    q = np.zeros((c, hq, d))
    got = prefill(L, table, pool, start, q, scale, splits)
    kk, vv = O.read(pool, L, table[0], n)
    ref, _, mass = O.attend(kk, vv, q, scale, start + 1 + np.arange(c))
    top = np.abs(vv).max() / start
    assert (np.abs(got - ref) <= C.out_bound(ref, mass, n, top)).all()


# --------------------------------------------------------------------------
# queries whose elements differ by many powers of two
# --------------------------------------------------------------------------
@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("far", [8, 10, 12, 13, 15, 17])
def test_prefill_of_queries_with_an_outlier(d, far):
    """One channel 2^far times the others, where the keys are zero, so that the others alone make the scores.  Elements
    within 2^13 of a row's largest enter exactly, smaller ones with an error of at most 2^-21 of it."""
    rng = np.random.default_rng(far)
    hq, hkv, start, c = 4, 2, 300, 40
    n, G = start + c, 2
    L = O.Layout(hkv, 64, d)
    table, pages = C.tables(rng, [-(-n // 64)])
    pool = O.new_pool(L, pages, 0xFF)
    k, v = rng.standard_normal((n, hkv, d)), C.rows(rng, n, hkv, d)
    k[:, :, 5] = 0
    k = torch.from_numpy(k).bfloat16().double().numpy()
    O.append(pool, L, table, [0], np.array([0, n]), k, v)
    # magnitudes in [1, 2) and the outlier 2^far: scores of the size that a softmax meets, times 4 so that few
    # positions carry each row
    q = (1 + rng.random((c, hq, d))) * rng.choice([-1.0, 1.0], (c, hq, d))
    q[:, :, 5] = 2.0 ** far
    q = torch.from_numpy(q).bfloat16().double().numpy()
    scale = float(np.float32(4 / math.sqrt(d)))
    got = prefill(L, table, pool, start, q, scale)
    kk, vv = O.read(pool, L, table[0], n)
    ref, w, mass = O.attend(kk, vv, q, scale, start + 1 + np.arange(c))
    rest = np.delete(np.arange(d), 5)
    for h in range(hq):
        # a score's error: the elements' own, and 2^-18 of the sum of |q k| for the products' fp32 sums; a weight is
        # off by its score's error and the largest of its row's
        off = 0.0 if far <= 13 else 2.0 ** -21 * 2.0 ** far
        ka = np.abs(kk[:, h // G][:, rest])
        e = (off * ka.sum(-1)[None] + 2.0 ** -18 * (np.abs(q[:, h][:, rest]) @ ka.T)) * scale
        # the elements' errors are of either sign and differ from each other: their sum over d of them stays below
        # 8 sqrt(d) of one's for all of these rows and positions, and max|k|
        if off:
            e = np.minimum(e, (off * 8 * math.sqrt(d) * ka.max() + 2.0 ** -18 * 4 * d * ka.max()) * scale)
        slack = 2 * e.max(-1)[:, None]
        top = (w[:, h].max(0)[:, None] * np.abs(vv[:, h // G])).max()
        bound = C.out_bound(ref[:, h], mass[:, h], n, top) + mass[:, h] * slack + n * top * 448 * 2.0 ** -25
        assert (np.abs(got[:, h] - ref[:, h]) <= bound).all(), float((np.abs(got[:, h] - ref[:, h]) / bound).max())


@pytest.mark.parametrize("qscale", [2.0 ** -60, 2.0 ** 20])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 128), (6, 1, 256)])
def test_prefill_of_scaled_queries(qscale, hq, hkv, d):
    """Queries far from 8 and 16 bits' ranges, each row by a power of two of its own, under a softmax scale to match."""
    rng = np.random.default_rng(d)
    start, c = 300, 40
    n = start + c
    L, table, pool = C.filled(rng, hkv, 64, d, [n])
    q = queries(rng, c, hq, d) * 2.0 ** rng.integers(-6, 3, (c, hq, 1)) * qscale
    scale = float(np.float32(1 / math.sqrt(d) / qscale))
    got = prefill(L, table, pool, start, q, scale)
    kk, vv = O.read(pool, L, table[0], n)
    ref, w, mass = O.attend(kk, vv, q, scale, start + 1 + np.arange(c))
    for h in range(hq):
        # a score's error: 2^-21 of the row's largest for each element that lies below 2^-13 of it, and 2^-18 of the
        # sum of |q k| for the fp32 sums
        ka = np.abs(kk[:, h * hkv // hq])
        e = (2.0 ** -21 * np.abs(q[:, h]).max(-1)[:, None] * ka.sum(-1)[None] + 2.0 ** -18 * np.abs(q[:, h]) @ ka.T) * scale
        top = (w[:, h].max(0)[:, None] * np.abs(vv[:, h * hkv // hq])).max()
        bound = (C.out_bound(ref[:, h], mass[:, h], n, top) + mass[:, h] * 2 * e.max(-1)[:, None] +
                 n * top * 448 * 2.0 ** -25)
        assert (np.abs(got[:, h] - ref[:, h]) <= bound).all(), float((np.abs(got[:, h] - ref[:, h]) / bound).max())


@pytest.mark.parametrize("hq,hkv,d,p,start,c,splits", [(4, 2, 128, 64, 250, 150, 1), (6, 1, 256, 128, 0, 130, 1),
                                                       (12, 2, 256, 64, 500, 90, 3), (1, 1, 128, 64, 63, 300, 1),
                                                       (8, 1, 128, 256, 700, 40, 4)])
def test_prefill_of_values_that_are_no_numbers(hq, hkv, d, p, start, c, splits):
    """NaN among the values of a position reaches the channel it lies in, of the queries that see the position, and
    nothing else: not the chunk's queries before it."""
    rng = np.random.default_rng(c)
    n = start + c
    L, table, pool = C.filled(rng, hkv, p, d, [n])
    q = queries(rng, c, hq, d)
    want = prefill(L, table, pool, start, q, 0.1, splits)
    assert np.isfinite(want).all()
    hit = np.zeros((c, hkv, d), dtype=bool)
    places = [(start + c - 1, 0, 5), (start + c // 2, 0, d - 1), (start + c // 2, hkv - 1, d // 2),
              (start + 1, hkv - 1, 17), (start + 33, 0, d // 2 - 1), (start + 33, 0, 0), (start, 0, 64)]
    if start > 64:
        places.append((start - 40, hkv - 1, 3))           # seen by all of the chunk
    for t, h, j in places:
        pool[table[0, t // p], ((hkv + h) * p + t % p) * d + j] = (0x7F, 0xFF)[t % 2]
        hit[max(t - start, 0):, h, j] = True
    hit = np.repeat(hit, hq // hkv, 1)
    got = prefill(L, table, pool, start, q, 0.1, splits)
    assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], want[~hit])


def test_prefill_of_values_that_are_no_numbers_in_a_divided_wave():
    """The same where the chunk's first rows have their histories in parts, and without a mask."""
    rng = np.random.default_rng(9)
    hq, hkv, d, p, start, c = 24, 4, 256, 256, 3400, 840
    pages = -(-(start + c) // p)
    g = jf.KVPool.allocate(pages, p, hkv, d, format=jf.JF_FMT_E4M3_B32)
    order = rng.permutation(pages)
    table = C.ints(order[None])
    torch.manual_seed(2)
    x = [torch.randn(start + c, hkv, d, device=DEV).bfloat16() for _ in range(2)]
    jf.jf_kv8_append(g, table, C.ints([0]), C.ints([0, start + c]), *x)
    q = torch.randn(c, hq, d, device=DEV).bfloat16()
    ws = jf.prefill_chunk_workspace(g, start, c, hq)
    outs = {}
    for poison in (False, True):
        if poison:
            hit = torch.zeros(c, hkv, d, dtype=torch.bool, device=DEV)
            for t, h, j in ((start + 1, 0, 7), (start + 20, 3, 200), (start + 839, 1, 0), (start + 400, 2, 127)):
                g.data[int(order[t // p]), ((hkv + h) * p + t % p) * d + j] = 0x7F
                hit[t - start:, h, j] = True
        for causal in (True, False):
            out = torch.full_like(q, 7.0)
            jf.jf_prefill_chunk_attn(g, table[0], q, start, 1 / 16, causal, out, ws)
            assert jf.workspace_status(ws) == 0
            outs[poison, causal] = out
    for causal in (True, False):
        bad = (hit if causal else hit.any(0, keepdim=True).expand_as(hit)).repeat_interleave(hq // hkv, 1)
        assert torch.isnan(outs[True, causal][bad]).all()
        assert torch.equal(outs[True, causal][~bad], outs[False, causal][~bad])
