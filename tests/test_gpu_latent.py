"""The latent cache on the GPU: append and read bit for bit, attention against the fp64 definitions."""
import math

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import latent as O
from tests import latent_cases as T
from tests.latent_cases import f64, gpu, ints

pytestmark = pytest.mark.gpu
DEV_PAGE, DEV_POS = 1, 2


# ---- append and read ------------------------------------------------------------------------
def appended(pool, table, start, off, x, P):
    """The fp64 pool after an append."""
    pool = pool.copy()
    for b in range(len(start)):
        t = start[b] + np.arange(off[b + 1] - off[b])
        pool[table[b, t // P], t % P] = x[off[b]:off[b + 1]]
    return pool


@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("P,start,n", [(64, [0], [1]), (64, [63, 0, 64], [2, 0, 65]), (128, [5, 1000, 127], [300, 1, 1]),
                                       (256, [0, 255, 256, 511], [0, 1, 257, 0])])
def test_append_and_read_back(R, P, start, n):
    rng = np.random.default_rng(R + P)
    table, pool = T.filled(rng, R, P, [s + m for s, m in zip(start, n)])
    pool = T.bf16(rng.standard_normal(pool.shape))
    off = np.concatenate([[0], np.cumsum(n)])
    total = int(off[-1])
    x = T.rows(rng, total + 3, R)                      # three rows of no request
    g, err = T.gpu_pool(pool), ints([0])
    rows = gpu(x)
    jf.jf_latent_append(g, ints(table), ints(start), ints(off), rows[:, :R], rows[:, R:], err)
    want = appended(pool, table, start, off, x, P)
    got = f64(g.data.view(torch.bfloat16).view(pool.shape))
    assert np.array_equal(got, want) and int(err) == 0
    back = torch.full((total + 3, R + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    rot = torch.full((total + 3, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    jf.jf_latent_read(g, ints(table), ints(start), ints(off), back[:, :R], rot, err)
    assert np.array_equal(f64(back)[:total, :R], x[:total, :R]) and np.array_equal(f64(rot)[:total], x[:total, R:])
    assert (back[total:] == 7).all() and (rot[total:] == 7).all() and (back[:, R:] == 7).all() and int(err) == 0


def test_append_skips_and_flags_what_does_not_fit():
    rng = np.random.default_rng(7)
    R, P = 256, 64
    pool = T.bf16(rng.standard_normal((4, P, R + 64)))
    table = np.array([[0, 9], [1, -1], [2, 3], [2, 3]], dtype=np.int32)
    x = T.rows(rng, 12, R)
    rows = gpu(x)
    # request 0 runs into a page outside the pool, 1 fits, 2 runs past its table row, 3 starts below 0
    g, err = T.gpu_pool(pool), ints([0])
    jf.jf_latent_append(g, ints(table), ints([62, 10, 126, -1]), ints([0, 4, 6, 9, 12]), rows[:, :R], rows[:, R:], err)
    want = pool.copy()
    want[0, 62:] = x[:2]
    want[1, 10:12] = x[4:6]
    assert np.array_equal(f64(g.data.view(torch.bfloat16).view(pool.shape)), want)
    assert int(err) == DEV_PAGE | DEV_POS
    err.zero_()
    back, rot = torch.full((12, R), 7.0, device="cuda").bfloat16(), torch.full((12, 64), 7.0, device="cuda").bfloat16()
    jf.jf_latent_read(g, ints(table), ints([62, 10, 126, -1]), ints([0, 4, 6, 9, 12]), back, rot, err)
    assert int(err) == DEV_PAGE | DEV_POS
    left = [2, 3] + list(range(6, 12))
    assert (back[left] == 7).all() and (rot[left] == 7).all()
    assert np.array_equal(f64(back)[[0, 1, 4, 5]], x[[0, 1, 4, 5], :R])
    # a request without rows is checked too
    err.zero_()
    jf.jf_latent_append(g, ints(table[:2]), ints([0, 1000]), ints([0, 1, 1]), rows[:1, :R], rows[:1, R:], err)
    assert int(err) == DEV_POS


def test_pages_far_into_a_large_pool():
    """A row's place passes 2^32 bytes."""
    R, P, pages = 512, 256, (1 << 32) // (256 * 576 * 2) + 40
    g = jf.KVPool.allocate(pages, P, 1, R + 64, format=jf.JF_FMT_LATENT16, fill=None)
    rng = np.random.default_rng(8)
    n = 300
    x = T.rows(rng, n, R)
    table, rows, err = ints([[pages - 1, pages - 3]]), gpu(x), ints([0])
    jf.jf_latent_append(g, table, ints([0]), ints([0, n]), rows[:, :R], rows[:, R:], err)
    back, rot = torch.empty(n, R, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 64, dtype=torch.bfloat16, device="cuda")
    jf.jf_latent_read(g, table, ints([0]), ints([0, n]), back, rot, err)
    assert int(err) == 0 and np.array_equal(f64(back), x[:, :R]) and np.array_equal(f64(rot), x[:, R:])
    q = T.queries(rng, 1, 3, R)
    out, ws = torch.empty(1, 3, R, dtype=torch.bfloat16, device="cuda"), jf.latent_decode_workspace(1, 3, R)
    jf.jf_latent_decode_attn(g, table, ints([n]), gpu(q), T.SCALE, out, ws)
    check(out[0], q[0], x, T.SCALE)


# ---- decode ---------------------------------------------------------------------------------
def check(out, q, kv, scale, R=None):
    ref, mass = O.decode(q, kv, scale)
    bound = T.decode_bound(ref, mass, T.score_error(q, kv, scale, kv.shape[1]))
    got = f64(out)
    assert got.shape == ref.shape
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (bad.sum(), np.abs(got - ref).max(), np.argwhere(bad)[:3])


def run_decode(table, pool, ctx, q, scale, ws=None):
    B, H, d = q.shape
    out = torch.full((B, H, d - 64), float("nan"), device="cuda").bfloat16()
    ws = jf.latent_decode_workspace(B, H, d - 64) if ws is None else ws
    jf.jf_latent_decode_attn(T.gpu_pool(pool), ints(table), ints(ctx), gpu(q), scale, out, ws)
    return out, jf.workspace_status(ws)


CTX = [[1], [2, 0], [63, 64, 65], [127, 128, 129, 0, 1], [1000, 3, 257, 640], [20000]]


@pytest.mark.parametrize("ctx", CTX, ids=str)
@pytest.mark.parametrize("R,H,P", [(512, 16, 64), (512, 1, 256), (256, 20, 128), (512, 128, 128), (256, 65, 64), (512, 130, 64)])
def test_decode(R, H, P, ctx):
    rng = np.random.default_rng(R + H + P + sum(ctx))
    table, pool = T.filled(rng, R, P, ctx)
    q = T.queries(rng, len(ctx), H, R)
    out, st = run_decode(table, pool, ctx, q, T.SCALE)
    assert st == 0
    for b, n in enumerate(ctx):
        check(out[b], q[b], O.gather(pool, table[b], n), T.SCALE)


def test_decode_of_many_requests():
    rng = np.random.default_rng(11)
    ctx = list(rng.integers(0, 400, 300))
    table, pool = T.filled(rng, 256, 64, ctx)
    q = T.queries(rng, 300, 8, 256)
    out, st = run_decode(table, pool, ctx, q, T.SCALE)
    assert st == 0
    for b, n in enumerate(ctx):
        check(out[b], q[b], O.gather(pool, table[b], n), T.SCALE)


def test_more_requests_than_threads():
    rng = np.random.default_rng(12)
    ctx = [int(n) for n in rng.integers(0, 130, 1500)]
    ctx[700], ctx[1499] = 20000, 3000
    table, pool = T.filled(rng, 256, 64, ctx)
    q = T.queries(rng, 1500, 4, 256)
    out, st = run_decode(table, pool, ctx, q, T.SCALE)
    assert st == 0
    for b, n in enumerate(ctx):
        check(out[b], q[b], O.gather(pool, table[b], n), T.SCALE)
    off, plens = [0, 1, 300, 300, 1100, 1500], [1, 200, 64, 5000, 0]
    both, pool = T.filled(rng, 256, 64, plens + ctx)
    out, st = run_prefix(pool, both[:5], plens, off, both[5:], ctx, q, T.SCALE)
    assert st == 0
    for g in range(5):
        for b in range(off[g], off[g + 1]):
            kv = np.concatenate([O.gather(pool, both[g], plens[g]), O.gather(pool, both[5 + b], ctx[b])])
            check(out[b], q[b], kv, T.SCALE)


@pytest.mark.parametrize("R", [256, 512])
def test_decode_of_long_and_short_requests_in_turn(R):
    """A pair of CTAs that takes the end of one request, others whole and a long run of the next."""
    rng = np.random.default_rng(19)
    ctx = [9000, 100, 0, 4097, 64, 7000, 1, 200, 6400, 8191, 130, 5000, 12, 3000, 9999, 128]
    table, pool = T.filled(rng, R, 256, ctx)
    q = T.queries(rng, len(ctx), 16, R)
    out, st = run_decode(table, pool, ctx, q, T.SCALE)
    assert st == 0
    for b, n in enumerate(ctx):
        check(out[b], q[b], O.gather(pool, table[b], n), T.SCALE)


@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0, 30.0])
def test_decode_scales(scale):
    """Equal weights, a negative scale, and scores so large that one position takes all."""
    rng = np.random.default_rng(12)
    table, pool = T.filled(rng, 512, 64, [777])
    q = T.queries(rng, 1, 16, 512)
    out, st = run_decode(table, pool, [777], q, scale)
    assert st == 0
    check(out[0], q[0], O.gather(pool, table[0], 777), scale)


@pytest.mark.parametrize("up", [True, False])
def test_scores_that_grow_or_fall_along_the_positions(up):
    """The running maximum moves in every tile: scores from -600 to 600 (in units of 1), and back."""
    rng = np.random.default_rng(13)
    n, R = 1500, 512
    table, pool = T.filled(rng, R, 64, [n])
    ramp = np.linspace(-600, 600, n) if up else np.linspace(600, -600, n)
    t = np.arange(n)
    pool[table[0, t // 64], t % 64, R] = T.bf16(ramp / 8)
    q = T.queries(rng, 1, 20, R)
    q[:, :, R] = 8 / T.SCALE
    q = T.bf16(q)
    out, st = run_decode(table, pool, [n], q, T.SCALE)
    assert st == 0
    check(out[0], q[0], O.gather(pool, table[0], n), T.SCALE)


def test_a_row_of_nan_and_one_of_infinity():
    rng = np.random.default_rng(14)
    table, pool = T.filled(rng, 512, 64, [300])
    q = T.queries(rng, 1, 16, 512)
    clean, _ = run_decode(table, pool, [300], q, T.SCALE)
    q[0, 3, 5], q[0, 9, 7] = np.nan, np.inf
    out, st = run_decode(table, pool, [300], q, T.SCALE)
    assert st == 0
    assert torch.isnan(out[0, 3]).all() and torch.isnan(out[0, 9]).all()
    keep = [h for h in range(16) if h not in (3, 9)]
    assert torch.equal(out[0, keep], clean[0, keep])


def test_a_nan_position_reaches_its_request_alone():
    rng = np.random.default_rng(15)
    table, pool = T.filled(rng, 256, 64, [100, 200, 100])
    q = T.queries(rng, 3, 8, 256)
    clean, _ = run_decode(table, pool, [100, 200, 100], q, T.SCALE)
    pool[table[1, 2], 3, 4] = np.nan
    out, st = run_decode(table, pool, [100, 200, 100], q, T.SCALE)
    assert st == 0 and torch.isnan(out[1]).all() and torch.equal(out[[0, 2]], clean[[0, 2]])


def test_pages_and_lengths_outside():
    """Positions of a page outside the pool draw no weight; a length that does not fit counts as none."""
    rng = np.random.default_rng(16)
    ctx = [300, 200, 130]
    table, pool = T.filled(rng, 512, 64, ctx)
    q = T.queries(rng, 3, 16, 512)
    bad = table.copy()
    bad[0, 2], bad[2, 0], bad[2, 1], bad[2, 2] = len(pool), -1, 1 << 30, -(1 << 31)
    out, st = run_decode(bad, pool, ctx, q, T.SCALE)
    assert st == DEV_PAGE
    kv = O.gather(pool, table[0], 300)
    check(out[0], q[0], np.concatenate([kv[:128], kv[192:]]), T.SCALE)
    check(out[1], q[1], O.gather(pool, table[1], 200), T.SCALE)
    assert (out[2] == 0).all()
    width = table.shape[1] * 64
    out, st = run_decode(table, pool, [300, -1, width + 1], q, T.SCALE)
    assert st == DEV_POS and (out[1:] == 0).all()
    check(out[0], q[0], kv, T.SCALE)


def test_decode_repeats_bit_for_bit_and_any_batch_order():
    rng = np.random.default_rng(17)
    ctx = [5000, 1, 900, 0, 64]
    table, pool = T.filled(rng, 512, 64, ctx)
    q = T.queries(rng, 5, 16, 512)
    ws = jf.latent_decode_workspace(5, 16, 512)
    one, _ = run_decode(table, pool, ctx, q, T.SCALE, ws)
    two, _ = run_decode(table, pool, ctx, q, T.SCALE, ws)
    assert torch.equal(one, two)
    order = [4, 2, 3, 0, 1]
    three, _ = run_decode(table[order], pool, [ctx[i] for i in order], q[order], T.SCALE, ws)
    for i, b in enumerate(order):
        check(three[i], q[b], O.gather(pool, table[b], ctx[b]), T.SCALE)


def test_a_batch_that_holds_nothing_yet():
    rng = np.random.default_rng(20)
    table, pool = T.filled(rng, 512, 64, [0, 0, 0])
    q = T.queries(rng, 3, 16, 512)
    out, st = run_decode(table, pool, [0, 0, 0], q, T.SCALE)
    assert st == 0 and (out == 0).all()
    out, st = run_prefix(pool, table[:1], [0], [0, 2], table[1:], [0, 0], q[:2], T.SCALE)
    assert st == 0 and (out == 0).all()


def test_three_row_blocks_a_request():
    rng = np.random.default_rng(23)
    table, pool = T.filled(rng, 256, 128, [3000, 1, 700])
    q = T.queries(rng, 3, 300, 256)
    out, st = run_decode(table, pool, [3000, 1, 700], q, T.SCALE)
    assert st == 0
    for b, n in enumerate([3000, 1, 700]):
        check(out[b], q[b], O.gather(pool, table[b], n), T.SCALE)


def test_memory_at_any_16_byte_address():
    """A pool, queries, weights and outputs that begin 16 bytes past a line."""
    rng = np.random.default_rng(24)
    table, pool = T.filled(rng, 512, 64, [500])
    raw = torch.empty(pool.size * 2 + 16, dtype=torch.uint8, device="cuda")
    data = raw[16:].view(len(pool), -1)
    data.copy_(T.gpu_pool(pool).data)
    g = jf.KVPool(data, 64, 1, 576, format=jf.JF_FMT_LATENT16)

    def moved(t):
        buf = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
        buf[8:].copy_(t.flatten())
        return buf[8:].view(t.shape)

    q, w, q3 = T.queries(rng, 1, 16, 512), weights(rng, 2, 512), T.bf16(rng.standard_normal((100, 2, 192)))
    out, out3 = moved(torch.zeros(1, 16, 512).bfloat16().cuda()), moved(torch.zeros(100, 2, 128).bfloat16().cuda())
    jf.jf_latent_decode_attn(g, ints(table), ints([500]), moved(gpu(q)), T.SCALE, out, jf.latent_decode_workspace(1, 16, 512))
    check(out[0], q[0], O.gather(pool, table[0], 500), T.SCALE)
    jf.jf_latent_prefill_attn(g, ints(table[0]), moved(gpu(q3)), 400, moved(gpu(w[0])), moved(gpu(w[1])), T.SCALE, True, out3,
                              jf.latent_prefill_workspace(400, 100, 2))
    check_prefill(out3, q3, O.gather(pool, table[0], 500), 400, w, T.SCALE, True)


def test_draft_tokens_as_requests():
    """Four tokens of one request: the same page-table row, a context length each."""
    rng = np.random.default_rng(18)
    table, pool = T.filled(rng, 512, 128, [500])
    q = T.queries(rng, 4, 16, 512)
    ctx = [497, 498, 499, 500]
    out, st = run_decode(np.repeat(table, 4, 0), pool, ctx, q, T.SCALE)
    assert st == 0
    for b, n in enumerate(ctx):
        check(out[b], q[b], O.gather(pool, table[0], n), T.SCALE)


# ---- shared prefixes --------------------------------------------------------------------------
def run_prefix(pool, ptable, plens, off, table, ctx, q, scale, ws=None):
    B, H, d = q.shape
    out = torch.full((B, H, d - 64), float("nan"), device="cuda").bfloat16()
    ws = jf.latent_decode_workspace(B, H, d - 64, num_groups=len(plens)) if ws is None else ws
    jf.jf_latent_prefix_decode_attn(T.gpu_pool(pool), ints(ptable), ints(plens), off, ints(table), ints(ctx), gpu(q),
                                    scale, out, ws)
    return out, jf.workspace_status(ws)


@pytest.mark.parametrize("R,H,P,sizes,plens,ctx", [
    (512, 16, 64, [3], [100], [0, 1, 70]),
    (512, 16, 64, [1], [5000], [33]),
    (256, 8, 128, [4, 0, 2], [130, 64, 1], [0, 0, 5, 200, 64, 63]),
    (512, 128, 64, [2, 3], [0, 257], [1, 0, 0, 2, 300]),
    (512, 5, 256, [40], [700], list(range(40))),
    (256, 64, 64, [3, 1], [65, 4000], [64, 128, 0, 1]),
    (512, 20, 64, [7, 9], [3000, 129], [0] * 16),
    (512, 16, 128, [30, 2, 9], [9000, 4000, 6001], [700 * (i % 3) + i for i in range(41)]),
    (256, 200, 64, [2, 1], [300, 64], [10, 0, 130]),
    (512, 1024, 128, [1, 2], [1500, 129], [1, 700, 0]),
], ids=str)
def test_prefix_decode(R, H, P, sizes, plens, ctx):
    rng = np.random.default_rng(R + H + sum(plens) + sum(ctx))
    both, pool = T.filled(rng, R, P, plens + ctx)
    G, off = len(plens), np.concatenate([[0], np.cumsum(sizes)]).tolist()
    q = T.queries(rng, len(ctx), H, R)
    out, st = run_prefix(pool, both[:G], plens, off, both[G:], ctx, q, T.SCALE)
    assert st == 0
    for g in range(G):
        for b in range(off[g], off[g + 1]):
            kv = np.concatenate([O.gather(pool, both[g], plens[g]), O.gather(pool, both[G + b], ctx[b])])
            check(out[b], q[b], kv, T.SCALE)


def test_prefix_errors_stay_in_their_group():
    rng = np.random.default_rng(21)
    plens, ctx, sizes = [200, 200, 200], [10, 20, 30, 40, 50, 60], [2, 2, 2]
    both, pool = T.filled(rng, 512, 64, plens + ctx)
    q = T.queries(rng, 6, 16, 512)
    bad = both.copy()
    bad[0, 1], bad[5, 0] = -1, len(pool)       # a page of group 0's prefix, and request 2's only page
    pl = [200, 200, both.shape[1] * 64 + 1]
    out, st = run_prefix(pool, bad[:3], pl, [0, 2, 4, 6], bad[3:], ctx, q, T.SCALE)
    assert st == DEV_PAGE | DEV_POS
    pre = [O.gather(pool, both[g], 200) for g in range(3)]
    own = [O.gather(pool, both[3 + b], n) for b, n in enumerate(ctx)]
    for b in (0, 1):
        check(out[b], q[b], np.concatenate([pre[0][:64], pre[0][128:], own[b]]), T.SCALE)
    check(out[2], q[2], pre[1], T.SCALE)
    check(out[3], q[3], np.concatenate([pre[1], own[3]]), T.SCALE)
    for b in (4, 5):
        check(out[b], q[b], own[b], T.SCALE)


def test_a_prefix_of_extreme_scores_beside_ordinary_ones():
    """One side's maximum far above the other's: the smaller side draws nothing."""
    rng = np.random.default_rng(22)
    both, pool = T.filled(rng, 512, 64, [500, 100, 100])
    t = np.arange(500)
    for sign in (1, -1):
        pool[both[0, t // 64], t % 64, 512] = sign * 50.0
        q = T.queries(rng, 2, 16, 512)
        q[:, :, 512] = 100.0
        out, st = run_prefix(pool, both[:1], [500], [0, 2], both[1:], [100, 100], q, T.SCALE)
        assert st == 0
        for b in range(2):
            check(out[b], q[b], np.concatenate([O.gather(pool, both[0], 500), O.gather(pool, both[1 + b], 100)]), T.SCALE)


# ---- prefill ----------------------------------------------------------------------------------
def weights(rng, H, R):
    return T.bf16(rng.standard_normal((2, H, 128, R)) / math.sqrt(1.65 * R))


def run_prefill(table_row, pool, q, q_start, w, scale, causal, ws=None):
    C, H, _ = q.shape
    out = torch.full((C, H, 128), float("nan"), device="cuda").bfloat16()
    ws = jf.latent_prefill_workspace(q_start, C, H) if ws is None else ws
    jf.jf_latent_prefill_attn(T.gpu_pool(pool), ints(table_row), gpu(q), q_start, gpu(w[0]), gpu(w[1]), scale, causal, out, ws)
    return out, jf.workspace_status(ws)


def check_prefill(out, q, kv, q_start, w, scale, causal, rows=None):
    ref, mass, reach = O.prefill(q, kv, q_start, w[0], w[1], scale, causal)
    # scores: keys off by 2^-8 of each channel and sums of 192 and R products in fp32 (a sum that cuts off:
    # 2^-23 an addition); values and weights by 2^-11 of each, or, below 2^-14 of a value and 2^-24 of the
    # largest weight, by 2^-25 and 2^-34 of it
    width = 192 + kv.shape[1]
    err = abs(scale) * reach[..., None] * (2.0 ** -8 + width * 2.0 ** -23)
    top = max(np.abs(O.expand(kv, w[0][h], w[1][h])[1]).max() for h in range(q.shape[1]))
    bound = (np.abs(ref) * 2.0 ** -8 + mass * (2.0 ** -10 + 2.0 ** -19 + np.expm1(2 * err)) + 2.0 ** -25
             + len(kv) * top * 2.0 ** -34)
    got = f64(out)
    pick = slice(None) if rows is None else rows
    bad = ~(np.abs(got - ref) <= bound)[pick]
    assert not bad.any(), (bad.sum(), np.abs(got - ref)[pick].max(), np.argwhere(bad)[:3])
    # roundings of either sign average out: the mean error stays below half a step of a typical term
    assert np.abs(got - ref)[pick].mean() <= 2.0 ** -8 * mass[pick].mean() + 2.0 ** -25


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("R,H,P,q_start,C", [(512, 1, 64, 0, 1), (512, 2, 64, 0, 130), (256, 3, 128, 63, 65), (512, 4, 256, 1, 257),
                                             (512, 16, 64, 1001, 77), (256, 1, 64, 5000, 3), (512, 2, 128, 127, 300),
                                             (512, 33, 64, 64, 64)])
def test_prefill(R, H, P, q_start, C, causal):
    rng = np.random.default_rng(R + H + q_start + C)
    n = q_start + C
    table, pool = T.filled(rng, R, P, [n])
    q, w = T.bf16(rng.standard_normal((C, H, 192))), weights(rng, H, R)
    out, st = run_prefill(table[0], pool, q, q_start, w, T.SCALE, causal)
    assert st == 0
    check_prefill(out, q, O.gather(pool, table[0], n), q_start, w, T.SCALE, causal)


@pytest.mark.parametrize("R,H,q_start,C,causal", [(256, 128, 0, 1, True), (256, 128, 0, 130, True), (512, 128, 300, 100, True),
                                                  (256, 64, 0, 1100, True), (256, 100, 120, 400, False)])
def test_prefill_of_many_heads(R, H, q_start, C, causal):
    """Several items for every pair of CTAs, one after the other, of one tile and of more."""
    rng = np.random.default_rng(R + H + C)
    n = q_start + C
    table, pool = T.filled(rng, R, 64, [n])
    q, w = T.bf16(rng.standard_normal((C, H, 192))), weights(rng, H, R)
    out, st = run_prefill(table[0], pool, q, q_start, w, T.SCALE, causal)
    assert st == 0
    kv = O.gather(pool, table[0], n)
    for h in range(0, H, 3):
        check_prefill(out[:, h:h + 1], q[:, h:h + 1], kv, q_start, w[:, h:h + 1], T.SCALE, causal)


def test_short_prefills_back_to_back():
    """Chunks too short to be divided, one after the other through one workspace: each call's expansion
    writes over the keys and values that the attention before it reads."""
    rng = np.random.default_rng(39)
    R, H, C = 512, 8, 40
    table, pool = T.filled(rng, R, 64, [C] * 12)
    g, w = T.gpu_pool(pool), weights(rng, H, R)
    wk, wv, ws = gpu(w[0]), gpu(w[1]), jf.latent_prefill_workspace(0, C, H)
    qs = [T.bf16(rng.standard_normal((C, H, 192))) for _ in range(12)]
    gq, rows = [gpu(q) for q in qs], [ints(table[b]) for b in range(12)]
    outs = [torch.zeros(C, H, 128, dtype=torch.bfloat16, device="cuda") for _ in range(12)]
    after = []
    torch.cuda.synchronize()
    for b in range(12):
        jf.jf_latent_prefill_attn(g, rows[b], gq[b], 0, wk, wv, T.SCALE, True, outs[b], ws)
        after.append(outs[b].clone())
    torch.cuda.synchronize()
    assert jf.workspace_status(ws) == 0
    for b in range(12):
        assert torch.equal(after[b], outs[b])
        check_prefill(outs[b], qs[b], O.gather(pool, table[b], C), 0, w, T.SCALE, True)


def test_prefill_in_several_passes():
    """More heads than the workspace holds keys and values of."""
    rng = np.random.default_rng(38)
    C, H, R = 4000, 60, 256
    table, pool = T.filled(rng, R, 256, [C])
    q, w = T.bf16(rng.standard_normal((C, H, 192))), weights(rng, H, R)
    assert jf.jf_latent_prefill_workspace_bytes(0, C, H) < H * 4096 * 512
    out, st = run_prefill(table[0], pool, q, 0, w, T.SCALE, True)
    assert st == 0
    kv = O.gather(pool, table[0], C)
    for h in (0, 29, 30, 59):
        check_prefill(out[:, h:h + 1], q[:, h:h + 1], kv, 0, w[:, h:h + 1], T.SCALE, True)


@pytest.mark.parametrize("scale", [0.0, -0.05, 3.0])
def test_prefill_scales(scale):
    rng = np.random.default_rng(31)
    table, pool = T.filled(rng, 512, 64, [400])
    q, w = T.bf16(rng.standard_normal((200, 2, 192))), weights(rng, 2, 512)
    out, st = run_prefill(table[0], pool, q, 200, w, scale, True)
    assert st == 0
    check_prefill(out, q, O.gather(pool, table[0], 400), 200, w, scale, True)


@pytest.mark.parametrize("up", [True, False])
def test_prefill_of_scores_that_grow_or_fall(up):
    rng = np.random.default_rng(32)
    n, R = 900, 512
    table, pool = T.filled(rng, R, 64, [n])
    ramp = np.linspace(-300, 300, n) * (1 if up else -1)
    t = np.arange(n)
    pool[table[0, t // 64], t % 64, R] = T.bf16(ramp / 8)
    q, w = T.bf16(rng.standard_normal((150, 2, 192))), weights(rng, 2, R)
    q[:, :, 128] = T.bf16(np.array([8 / T.SCALE]))[0]
    out, st = run_prefill(table[0], pool, q, n - 150, w, T.SCALE, True)
    assert st == 0
    check_prefill(out, q, O.gather(pool, table[0], n), n - 150, w, T.SCALE, True)


@pytest.mark.parametrize("what", [np.nan, np.inf])
def test_a_value_that_is_not_finite_reaches_the_queries_that_see_it_alone(what):
    rng = np.random.default_rng(33)
    n, q_start = 300, 100
    table, pool = T.filled(rng, 512, 64, [n])
    q, w = T.bf16(rng.standard_normal((200, 3, 192))), weights(rng, 3, 512)
    at = 230
    kv = O.gather(pool, table[0], n)
    pool[table[0, at // 64], at % 64, 17] = what
    out, st = run_prefill(table[0], pool, q, q_start, w, T.SCALE, True)
    assert st == 0 and torch.isnan(out[at - q_start:]).all()
    check_prefill(out, q, kv, q_start, w, T.SCALE, True, rows=slice(0, at - q_start))


def test_a_value_past_fp16_is_flagged():
    rng = np.random.default_rng(36)
    table, pool = T.filled(rng, 256, 64, [200])
    q, w = T.bf16(rng.standard_normal((150, 3, 192))), weights(rng, 3, 256)
    w[1, 1] *= 2.0 ** 20
    out, st = run_prefill(table[0], pool, q, 50, w, T.SCALE, True)
    assert st == 16                                     # JF_DEV_ERR_RANGE
    keep = [0, 2]
    check_prefill(out[:, keep], q[:, keep], O.gather(pool, table[0], 200), 50, w[:, keep], T.SCALE, True)


@pytest.mark.parametrize("power", [-30, 13])
def test_small_and_large_values(power):
    """Values near either end of fp16: products of 2^-30 lose all but what 2^-25 leaves of them."""
    rng = np.random.default_rng(37)
    table, pool = T.filled(rng, 256, 64, [200])
    q, w = T.bf16(rng.standard_normal((150, 2, 192))), weights(rng, 2, 256)
    w[1] *= 2.0 ** power
    out, st = run_prefill(table[0], pool, q, 50, w, T.SCALE, True)
    assert st == 0
    check_prefill(out, q, O.gather(pool, table[0], 200), 50, w, T.SCALE, True)


def test_a_query_of_nan_stays_alone():
    rng = np.random.default_rng(34)
    table, pool = T.filled(rng, 256, 64, [200])
    q, w = T.bf16(rng.standard_normal((150, 2, 192))), weights(rng, 2, 256)
    clean, _ = run_prefill(table[0], pool, q, 50, w, T.SCALE, True)
    q[70, 1, 3] = np.nan
    out, _ = run_prefill(table[0], pool, q, 50, w, T.SCALE, True)
    assert torch.isnan(out[70, 1]).all()
    out[70, 1] = clean[70, 1]
    assert torch.equal(out, clean)


def test_prefill_flags_a_page_outside_the_pool():
    rng = np.random.default_rng(35)
    table, pool = T.filled(rng, 512, 64, [300])
    q, w = T.bf16(rng.standard_normal((150, 2, 192))), weights(rng, 2, 512)
    bad = table[0].copy()
    bad[4] = len(pool)                                  # positions 256 .. 299
    out, st = run_prefill(bad, pool, q, 150, w, T.SCALE, True)
    assert st == DEV_PAGE
    check_prefill(out, q, O.gather(pool, table[0], 300), 150, w, T.SCALE, True, rows=slice(0, 106))


def test_an_empty_chunk_is_a_no_op():
    pool = jf.KVPool.allocate(2, 64, 1, 576, format=jf.JF_FMT_LATENT16)
    q, w = torch.zeros(0, 2, 192, device="cuda").bfloat16(), torch.zeros(2, 128, 512, device="cuda").bfloat16()
    jf.jf_latent_prefill_attn(pool, ints([0, 1]), q, 10, w, w, 0.1, True, q[..., :128].contiguous(),
                              jf.latent_prefill_workspace(10, 0, 2))


# ---- together, captured, on other streams -----------------------------------------------------
def test_a_prompt_its_branches_and_their_tokens():
    """Append and prefill a prompt in chunks, branch it, and decode tokens of every branch in the absorbed form, each
    appended first; the same outputs from the definitions on the dense rows.  Pages copied out and back hold the same."""
    rng = np.random.default_rng(41)
    R, H, P, n, branches = 512, 4, 64, 230, 3
    w = weights(rng, H, R)
    x = T.rows(rng, n, R)
    pool = jf.KVPool.allocate(16, P, 1, R + 64, format=jf.JF_FMT_LATENT16, fill=0xFF)
    table = ints([[7, 3, 11, 0]])
    err, rows = ints([0]), gpu(x)
    for a, b in ((0, 100), (100, 230)):
        jf.jf_latent_append(pool, table, ints([a]), ints([0, b - a]), rows[a:b, :R], rows[a:b, R:], err)
        q = T.bf16(rng.standard_normal((b - a, H, 192)))
        out = torch.empty(b - a, H, 128, dtype=torch.bfloat16, device="cuda")
        ws = jf.latent_prefill_workspace(a, b - a, H)
        jf.jf_latent_prefill_attn(pool, table[0], gpu(q), a, gpu(w[0]), gpu(w[1]), T.SCALE, True, out, ws)
        assert jf.workspace_status(ws) == 0
        check_prefill(out, q, x[:b], a, w, T.SCALE, True)
    blob = torch.empty(4 * P * (R + 64) * 2, dtype=torch.uint8, device="cuda")
    jf.jf_kv_checkpoint(pool, table[0], 4, blob, err)
    pool.data[[7, 3, 11, 0]] = 0
    jf.jf_kv_restore(pool, table[0], 4, blob, err)
    own = ints([[1], [2], [4]])
    held = [np.zeros((0, R + 64)) for _ in range(branches)]
    ws = jf.latent_decode_workspace(branches, H, R, num_groups=1)
    for step in range(3):
        new = T.rows(rng, branches, R)
        r = gpu(new)
        jf.jf_latent_append(pool, own, ints([step] * branches), ints(range(branches + 1)), r[:, :R], r[:, R:], err)
        q = T.queries(rng, branches, H, R)
        out = torch.empty(branches, H, R, dtype=torch.bfloat16, device="cuda")
        jf.jf_latent_prefix_decode_attn(pool, table, ints([n]), [0, branches], own, ints([step + 1] * branches), gpu(q),
                                        T.SCALE, out, ws)
        assert jf.workspace_status(ws) == 0 and int(err) == 0
        for b in range(branches):
            held[b] = np.concatenate([held[b], new[b:b + 1]])
            check(out[b], q[b], np.concatenate([x, held[b]]), T.SCALE)


@pytest.mark.parametrize("op", ["decode", "prefix", "prefill"])
def test_captured_and_replayed_with_other_lengths(op):
    rng = np.random.default_rng(42)
    R, H, P = 512, 16, 64
    both, pool = T.filled(rng, R, P, [600, 400, 300])
    g, q = T.gpu_pool(pool), T.queries(rng, 2, H, R)
    q3, w = T.bf16(rng.standard_normal((90, 2, 192))), weights(rng, 2, R)
    lens, plen = ints([400, 300]), ints([600])
    out = torch.zeros(2, H, R, dtype=torch.bfloat16, device="cuda")
    out3 = torch.zeros(90, 2, 128, dtype=torch.bfloat16, device="cuda")
    qg, q3g, wk, wv, tb, pt = gpu(q), gpu(q3), gpu(w[0]), gpu(w[1]), ints(both[1:]), ints(both[:1])
    ws = (jf.latent_prefill_workspace(300, 90, 2) if op == "prefill" else
          jf.latent_decode_workspace(2, H, R, num_groups=1 if op == "prefix" else 0))

    def call():
        if op == "decode":
            jf.jf_latent_decode_attn(g, tb, lens, qg, T.SCALE, out, ws)
        elif op == "prefix":
            jf.jf_latent_prefix_decode_attn(g, pt, plen, [0, 2], tb, lens, qg, T.SCALE, out, ws)
        else:
            jf.jf_latent_prefill_attn(g, pt[0], q3g, 300, wk, wv, T.SCALE, True, out3, ws)

    def right(ctx, n):
        pre = O.gather(pool, both[0], n)
        if op == "prefill":
            check_prefill(out3, q3, O.gather(pool, both[0], 390), 300, w, T.SCALE, True)
            return
        for b in range(2):
            own = O.gather(pool, both[1 + b], ctx[b])
            check(out[b], q[b], np.concatenate([pre, own]) if op == "prefix" else own, T.SCALE)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    right([400, 300], 600)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for ctx, n in (([400, 300], 600), ([1, 0], 599), ([65, 300], 1), ([400, 299], 0)):
        lens.copy_(ints(ctx))
        plen.copy_(ints([n]))
        out.zero_()
        out3.zero_()
        graph.replay()
        torch.cuda.synchronize()
        right(ctx, n)
    assert jf.workspace_status(ws) == 0


def test_two_calls_at_once_on_workspaces_of_their_own():
    rng = np.random.default_rng(43)
    table, pool = T.filled(rng, 512, 64, [9000, 8000])
    g, q = T.gpu_pool(pool), T.queries(rng, 2, 16, 512)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros(1, 16, 512, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    wss = [jf.latent_decode_workspace(1, 16, 512) for _ in range(2)]
    args = [(ints(table[b:b + 1]), ints([[9000, 8000][b]]), gpu(q[b:b + 1])) for b in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for b in range(2):
            jf.jf_latent_decode_attn(g, args[b][0], args[b][1], args[b][2], T.SCALE, outs[b], wss[b], stream=streams[b])
    torch.cuda.synchronize()
    for b in range(2):
        assert jf.workspace_status(wss[b]) == 0
        check(outs[b][0], q[b], O.gather(pool, table[b], [9000, 8000][b]), T.SCALE)
