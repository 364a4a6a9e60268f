"""The 8-bit block-scaled cache on the GPU against its fp64 oracle: append and read bit for bit, attention and
weights within bounds derived in kv8_cases."""
import math

import numpy as np
import pytest
import torch

import paper_2609_17475_gb300 as jf
from oracle import kv8 as O
from tests import kv8_cases as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def flag():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


def gpu_append(pool, table, start, offsets, k, v, err=None):
    err = flag() if err is None else err
    jf.jf_kv8_append(pool, C.ints(table), C.ints(start), C.ints(offsets), k, v, err)
    return err


# --------------------------------------------------------------------------
# append and read
# --------------------------------------------------------------------------
@pytest.mark.parametrize("hkv,d,p,start,count", [
    (2, 128, 64, [0], [1]),
    (1, 256, 64, [0], [257]),
    (4, 256, 256, [31, 0, 511], [1, 300, 2]),
    (3, 128, 128, [5, 64, 0, 95], [0, 32, 33, 161]),
    (2, 256, 128, [30], [4]),
    (1, 128, 256, list(range(0, 40)), [1] * 40),
])
def test_append_and_read_bit_for_bit(hkv, d, p, start, count):
    rng = np.random.default_rng(sum(start) + d)
    L, table, pool = C.filled(rng, hkv, p, d, start, extra=[-(-(s + c) // p) - -(-s // p) for s, c in zip(start, count)])
    off = np.concatenate([[0], np.cumsum(count)])
    n = int(off[-1])
    k, v = C.rows(rng, n, hkv, d), C.rows(rng, n, hkv, d)
    if n:
        k[rng.random(n) < 0.3] *= 16        # blocks that grow
        v[n // 2] = 0
    g = C.gpu_pool(L, pool.copy())
    err = gpu_append(g, table, start, off, C.bf16(k), C.bf16(v))
    O.append(pool, L, table, start, off, k, v)
    assert int(err) == 0
    assert np.array_equal(g.data.cpu().numpy(), pool)      # codes, scales, and every byte that is not theirs
    got = [torch.full((n, hkv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    jf.jf_kv8_read(g, C.ints(table), C.ints(start), C.ints(off), *got, err)
    for b, (s, c) in enumerate(zip(start, count)):
        ref = O.read(pool, L, table[b], s + c)
        for kind in range(2):
            x = got[kind][off[b]:off[b + 1]].double().cpu().numpy()
            assert np.array_equal(x, ref[kind][s:])


def test_append_row_by_row_and_again():
    """Rows one at a time through a growing block, and the same call twice: the oracle's bytes each time."""
    rng = np.random.default_rng(8)
    L = O.Layout(2, 64, 128)
    table = np.array([[2, 0]], dtype=np.int32)
    k, v = C.rows(rng, 70, 2, 128), C.rows(rng, 70, 2, 128)
    k[10:] *= 8
    k[20:] *= 64
    pool = O.new_pool(L, 3, 0x5A)
    g = C.gpu_pool(L, pool.copy())
    for i in range(70):
        for _ in range(2):
            err = gpu_append(g, table, [i], [0, 1], C.bf16(k[i:i + 1]), C.bf16(v[i:i + 1]))
        O.append(pool, L, table, [i], [0, 1], k[i:i + 1], v[i:i + 1])
    assert int(err) == 0 and np.array_equal(g.data.cpu().numpy(), pool)


def test_append_of_unusual_values():
    """NaN stays NaN and scales nothing; infinities and values past 448 * 2^40 saturate; zeros, signed zeros,
    subnormals and ties follow the definition."""
    L = O.Layout(1, 64, 128)
    x = np.zeros((7, 1, 128))
    x[0, 0, :4] = [1.0, -0.0, 2.0 ** -126, -2.0 ** -133]
    x[1] = np.linspace(-1, 1, 128)
    x[2, 0, :3] = [17.0, 19.0, 21.0]               # midpoints of codes 16, 18, 20, 22
    x = torch.from_numpy(x).bfloat16().double().numpy()
    y = x.copy()
    y[3, 0, 5], y[3, 0, 6], y[4, 0, 7] = np.nan, np.inf, -np.inf
    big = np.zeros((7, 1, 128))
    big[0, 0, :2] = [2.0 ** 120, -2.0 ** 49]
    big[1, 0, 0] = 448 * 2.0 ** 40
    for k, v in ((x, y), (y, big), (big, np.zeros_like(x))):
        pool = O.new_pool(L, 1, 0)
        g = C.gpu_pool(L, pool.copy())
        assert int(gpu_append(g, [[0]], [0], [0, 7], C.bf16(k), C.bf16(v))) == 0
        O.append(pool, L, [[0]], [0], [0, 7], k, v)
        assert np.array_equal(g.data.cpu().numpy(), pool)


def test_append_of_strided_rows_on_another_stream():
    """K and V inside one fused projection; a side stream, ordered by events."""
    rng = np.random.default_rng(9)
    hkv, d = 2, 128
    L = O.Layout(hkv, 64, d)
    qkv = torch.randn(50, 6 + 2 * hkv, d, device=DEV).bfloat16()
    k, v = qkv[:, 6:6 + hkv], qkv[:, 6 + hkv:]
    g = jf.KVPool.allocate(1, 64, hkv, d, format=jf.JF_FMT_E4M3_B32)
    assert g.page_bytes == L.page_bytes
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    back = torch.zeros(50, 2 * hkv, d, dtype=torch.bfloat16, device=DEV)
    with torch.cuda.stream(s):
        err = gpu_append(g, [[0]], [0], [0, 50], k, v)
        jf.jf_kv8_read(g, C.ints([[0]]), C.ints([0]), C.ints([0, 50]), back[:, :hkv], back[:, hkv:], err)
    torch.cuda.current_stream().wait_stream(s)
    pool = O.new_pool(L, 1, 0)
    O.append(pool, L, [[0]], [0], [0, 50], k.double().cpu().numpy(), v.double().cpu().numpy())
    assert int(err) == 0 and np.array_equal(g.data.cpu().numpy(), pool)
    ref = np.concatenate(O.read(pool, L, [0], 50), 1)
    assert np.array_equal(back.double().cpu().numpy(), ref)


def test_append_and_read_report_what_does_not_fit():
    """Positions past the table, bad offsets and bad pages are reported and skipped; the others are done."""
    rng = np.random.default_rng(10)
    L = O.Layout(1, 64, 128)
    k, v = C.rows(rng, 12, 1, 128), C.rows(rng, 12, 1, 128)
    table = np.array([[0, 1], [2, 9], [-1, 3], [4, 5]], dtype=np.int32)
    pos_bit, page_bit = jf.binding.JF_DEV_ERR_POSITION, jf.binding.JF_DEV_ERR_PAGE_ID
    for start, off, want, good in (
            ([126, 0, 64, 5], [0, 3, 6, 9, 12], pos_bit, [1, 2, 3]),      # request 0 ends at 129 > 128
            ([0, -1, 64, 5], [0, 3, 6, 9, 12], pos_bit, [0, 2, 3]),
            ([0, 64, 64, 5], [0, 3, 6, 9, 12], page_bit, [0, 2, 3]),      # request 1's page 9 of 6
            ([0, 0, 0, 5], [0, 3, 6, 9, 12], page_bit, [0, 1, 3]),        # request 2's page -1
            ([0, 0, 64, 5], [0, 3, 2, 9, 12], pos_bit, [0, 2, 3]),        # falling offsets
            ([0, 0, 64, 5], [0, 3, 6, 9, 13], pos_bit, [0, 1, 2])):       # past the rows
        pool = O.new_pool(L, 6, 0x11)
        g = C.gpu_pool(L, pool.copy())
        err = gpu_append(g, table, start, off, C.bf16(k), C.bf16(v))
        assert int(err) == want, (start, off)
        for b in good:
            O.append(pool, L, [table[b]], [start[b]], [off[b], off[b + 1]], k, v)
        assert np.array_equal(g.data.cpu().numpy(), pool), (start, off)
        if off == [0, 3, 6, 9, 12]:
            got = [torch.full((12, 1, 128), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            err = flag()
            jf.jf_kv8_read(g, C.ints(table), C.ints(start), C.ints(off), *got, err)
            assert int(err) == want
            for b in range(4):
                assert (got[0][off[b]:off[b + 1]] == 7.0).all().item() == (b not in good)


def test_offsets_past_32_bits():
    """Pages more than 4 GiB into a pool: append, read, decode and prefill give what a small pool gives."""
    rng = np.random.default_rng(11)
    hkv, d, p = 4, 256, 256
    L = O.Layout(hkv, p, d)
    pages = (5 << 30) // L.page_bytes
    far, near = np.array([[pages - 1, pages - 3]]), np.array([[0, 1]])
    n = 300
    k, v = C.bf16(C.rows(rng, n, hkv, d)), C.bf16(C.rows(rng, n, hkv, d))
    q = torch.randn(1, 8, d, device=DEV).bfloat16()
    qp = torch.randn(40, 8, d, device=DEV).bfloat16()
    res = []
    for count, table in ((pages, far), (2, near)):
        g = jf.KVPool.allocate(count, p, hkv, d, fill=None, format=jf.JF_FMT_E4M3_B32)
        err = gpu_append(g, table, [0], [0, n], k, v)
        back = [torch.zeros_like(k), torch.zeros_like(v)]
        jf.jf_kv8_read(g, C.ints(table), C.ints([0]), C.ints([0, n]), *back, err)
        out, ws = torch.zeros_like(q), jf.decode_workspace(1, 8, hkv, d, 4)
        jf.jf_paged_decode_attn(g, C.ints(table), C.ints([n]), q, 0.06, out, ws, 4)
        outp, wsp = torch.zeros_like(qp), torch.zeros(256, dtype=torch.uint8, device=DEV)
        jf.jf_prefill_chunk_attn(g, C.ints(table)[0], qp, n - 40, 0.06, True, outp, wsp)
        assert int(err) == 0 and jf.workspace_status(ws) == 0 and jf.workspace_status(wsp) == 0
        res.append(back + [out, outp])
        del g
    for a, b in zip(*res):
        assert torch.equal(a, b)


# --------------------------------------------------------------------------
# single-token attention, weights
# --------------------------------------------------------------------------
def decode(L, table, pool, ctx, q, scale, splits, w_in=None, weigh=False, stride=None):
    g = C.gpu_pool(L, pool)
    B, Hq, D = q.shape
    out = torch.full((B, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    if not weigh:
        ws = jf.decode_workspace(B, Hq, L.Hkv, D, splits)
        ws[256:] = 0xFF
        jf.jf_paged_decode_attn(g, C.ints(table), C.ints(ctx), C.bf16(q), scale, out, ws, splits)
        return out, None, jf.workspace_status(ws)
    stride = max(max(ctx), 1) if stride is None else stride
    ws = jf.decode_weights_workspace(B, Hq, L.Hkv, D, splits, stride)
    ws[256:] = 0xFF
    w = torch.full((B, L.Hkv, stride), -3.0, device=DEV)
    if w_in is not None:
        w_in = torch.from_numpy(w_in).to(DEV)
    jf.jf_paged_decode_weights_attn(g, C.ints(table), C.ints(ctx), C.bf16(q), scale, out, w_in, w, ws, splits)
    return out, w, jf.workspace_status(ws)


def check_decode(L, table, pool, ctx, q, scale, out, w=None, w_in=None):
    G = q.shape[1] // L.Hkv
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    for b, n in enumerate(ctx):
        k, v = O.read(pool, L, table[b], n)
        ref, p, mass = O.attend(k, v, q[b:b + 1], scale)
        top = max((p[0, h][:, None] * np.abs(v[:, h // G])).max(initial=0) for h in range(q.shape[1]))
        err = np.abs(got[b] - ref[0])
        bound = C.out_bound(ref[0], mass[0], n, top)
        assert (err <= bound).all(), (b, n, float((err - bound).max()))
        if w is None:
            continue
        gw = w[b].cpu().numpy()
        assert (gw[:, n:] == -3.0).all()            # not written past the context
        for h in range(L.Hkv):
            want = w_in[b, h, :n].astype(np.float64) if w_in is not None else np.zeros(n)
            add, slack = np.zeros(n), np.zeros(n)
            for g in range(G):
                hq = h * G + g
                # a score's error: D fp32 additions of products that are exact, 2^-23 of the sum of |q k| each at
                # most, and three roundings of the score; a weight's: its score's, the largest of its row's (in
                # the sum), and 2^-20 for the exponentials and the sum of n terms
                mag = np.abs(k[:, h]) @ np.abs(q[b, hq]) * scale
                d = 2.0 ** -23 * (L.D * mag / 16 + 4 * mag)
                add += p[0, hq]
                slack += p[0, hq] * (d + d.max(initial=0) + 2.0 ** -20) * 1.05
            bound = slack + 2.0 ** -23 * np.abs(want + add) + 2.0 ** -140
            err = np.abs(gw[h, :n] - (want + add))
            assert (err <= bound).all(), (b, h, float((err / bound).max()))


@pytest.mark.parametrize("hq,hkv,d,p,ctx,splits", [
    (8, 2, 128, 64, [1], 1),
    (8, 2, 128, 256, [4096], 76),
    (24, 4, 256, 256, [777, 1, 0, 33, 2049], 6),
    (6, 1, 256, 64, [15], 3),
    (8, 1, 128, 128, [16, 17, 31, 32, 47, 48, 49, 63, 64, 65, 127, 128, 129], 2),
    (4, 4, 256, 128, [1000], 9),
    (5, 5, 128, 64, [0, 0, 600], 4),
    (7, 1, 256, 256, [6000], 152),
    (14, 2, 128, 64, [191, 193, 4097, 2], 1),
    (3, 3, 256, 64, [0], 5),
])
@pytest.mark.parametrize("weigh", [False, True])
def test_decode(hq, hkv, d, p, ctx, splits, weigh):
    rng = np.random.default_rng(hq + d + sum(ctx))
    L, table, pool = C.filled(rng, hkv, p, d, ctx)          # every other byte 0xff: NaN codes, NaN scales
    q = torch.from_numpy(rng.standard_normal((len(ctx), hq, d))).bfloat16().double().numpy()
    scale = 1 / math.sqrt(d)
    w_in = rng.random((len(ctx), hkv, max(max(ctx), 1) + 3), dtype=np.float32) if weigh and len(ctx) > 1 else None
    stride = None if w_in is None else w_in.shape[2]
    out, w, status = decode(L, table, pool, ctx, q, scale, splits, w_in, weigh, stride)
    assert status == 0
    check_decode(L, table, pool, ctx, q, np.float32(scale).astype(np.float64), out, w, w_in)
    again = decode(L, table, pool, ctx, q, scale, splits, w_in, weigh, stride)
    assert torch.equal(out, again[0]) and (w is None or torch.equal(w, again[1]))


@pytest.mark.parametrize("spread", [8, 30])
@pytest.mark.parametrize("qscale", [1.0, 2.0 ** -60, 2.0 ** 20])
def test_decode_of_blocks_with_very_different_scales(spread, qscale):
    """V blocks from 2^-spread to 2^spread (K blocks likewise for V's sake only: their scores saturate the softmax),
    queries far from fp16's range: still within the bounds, which are relative to what each row attends."""
    rng = np.random.default_rng(spread)
    hq, hkv, d, p, ctx = 6, 2, 128, 64, [700, 95]
    L = O.Layout(hkv, p, d)
    table, pages = C.tables(rng, [11, 2])
    pool = O.new_pool(L, pages, 0xFF)
    off = [0, 700, 795]
    O.append(pool, L, table, [0, 0], off, C.rows(rng, 795, hkv, d), C.rows(rng, 795, hkv, d, spread))
    q = torch.from_numpy(rng.standard_normal((2, hq, d)) * qscale).bfloat16().double().numpy()
    scale = float(np.float32(1 / math.sqrt(d) / qscale))
    out, w, status = decode(L, table, pool, ctx, q, scale, 5, None, True)
    assert status == 0
    check_decode(L, table, pool, ctx, q, scale, out, w)


def test_decode_one_hot_and_flat_softmax():
    """A key that takes everything gives its V exactly; zero queries give the mean."""
    rng = np.random.default_rng(21)
    L, table, pool = C.filled(rng, 1, 64, 128, [500])
    k, v = O.read(pool, L, table[0], 500)
    q = np.zeros((1, 2, 128))
    q[0, 0] = torch.from_numpy(k[123, 0] * 64).bfloat16().double().numpy()
    out, w, status = decode(L, table, pool, [500], q, 1.0, 3, None, True)
    assert status == 0
    check_decode(L, table, pool, [500], q, 1.0, out, w)
    s = k[:, 0] @ q[0, 0]
    top = int(s.argmax())                       # the others are at least 2^-40 below it
    assert np.sort(s)[-2] < s[top] - 40
    assert np.array_equal(out[0, 0].double().cpu().numpy(), v[top, 0])
    rest = torch.ones(500, dtype=torch.bool, device=DEV)
    rest[top] = False
    assert abs(float(w[0, 0, top]) - 1.002) < 1e-6 and torch.allclose(
        w[0, 0, rest], torch.full((499,), 0.002, device=DEV), rtol=1e-5)


def test_weights_add_up_in_place_over_steps():
    rng = np.random.default_rng(22)
    ctx = [300, 70]
    L, table, pool = C.filled(rng, 2, 128, 128, ctx)
    g = C.gpu_pool(L, pool)
    w = torch.zeros(2, 2, 300, device=DEV)
    ws = jf.decode_weights_workspace(2, 8, 2, 128, 4, 300)
    total = [np.zeros((2, n)) for n in ctx]
    for _ in range(5):
        q = torch.from_numpy(rng.standard_normal((2, 8, 128))).bfloat16().double().numpy()
        out = torch.empty(2, 8, 128, dtype=torch.bfloat16, device=DEV)
        jf.jf_paged_decode_weights_attn(g, C.ints(table), C.ints(ctx), C.bf16(q), 0.1, out, w, w, ws, 4)
        for b, n in enumerate(ctx):
            p = O.attend(*O.read(pool, L, table[b], n), q[b:b + 1], 0.1)[1][0]
            total[b] += p.reshape(2, 4, n).sum(1)
    assert jf.workspace_status(ws) == 0
    for b, n in enumerate(ctx):
        assert np.allclose(w[b, :, :n].cpu().numpy(), total[b], rtol=1e-4, atol=1e-9)
        assert not w[b, :, n:].any()


def test_decode_reports_pages_and_lengths():
    """A page outside the pool drops its positions; a context past the table is cut to it; both are reported."""
    rng = np.random.default_rng(23)
    L, table, pool = C.filled(rng, 1, 64, 128, [200, 128])
    bad = table.copy()
    bad[0, 1], bad[1, 0] = -1, len(pool)
    q = torch.from_numpy(rng.standard_normal((2, 4, 128))).bfloat16().double().numpy()
    out, _, status = decode(L, bad, pool, [200, 128], q, 0.1, 3)
    assert status == jf.binding.JF_DEV_ERR_PAGE_ID
    for b, seen in ((0, np.r_[0:64, 128:200]), (1, np.r_[64:128])):
        k, v = O.read(pool, L, table[b], [200, 128][b])
        ref, p, mass = O.attend(k[seen], v[seen], q[b:b + 1], 0.1)
        err = np.abs(out[b].double().cpu().numpy() - ref[0])
        assert (err <= C.out_bound(ref[0], mass[0], 200, np.abs(v).max())).all()
    full = table[:, :2].copy()
    out, w, status = decode(L, full, pool, [200, 128], q, 0.1, 3, None, True, stride=256)
    assert status == jf.binding.JF_DEV_ERR_POSITION
    check_decode(L, full, pool, [128, 128], q, 0.1, out)
    out, _, status = decode(L, full, pool, [-5, 128], q, 0.1, 3)
    assert status == jf.binding.JF_DEV_ERR_POSITION and not out[0].any()
    # weights shorter than a context: reported, and nothing outside them is read or written
    out, w, status = decode(L, table, pool, [200, 128], q, 0.1, 3, None, True, stride=150)
    assert status == jf.binding.JF_DEV_ERR_POSITION
    check_decode(L, table, pool, [150, 128], q, 0.1, out, w)


def test_decode_in_a_graph_and_on_a_stream():
    """Append and attend captured once and replayed as positions advance."""
    rng = np.random.default_rng(24)
    hkv, d, p = 2, 128, 64
    L, table, pool = C.filled(rng, hkv, p, d, [60], extra=[1])
    g = C.gpu_pool(L, pool.copy())
    t, start, off = C.ints(table), C.ints([60]), C.ints([0, 1])
    ctx, err = C.ints([61]), flag()
    k, v, q = (torch.zeros(1, h, d, dtype=torch.bfloat16, device=DEV) for h in (hkv, hkv, 8))
    out, ws = torch.zeros_like(q), jf.decode_workspace(1, 8, hkv, d, 8)

    def step():
        jf.jf_kv8_append(g, t, start, off, k, v, err)
        jf.jf_paged_decode_attn(g, t, ctx, q, 0.1, out, ws, 8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(10):
        rows = [torch.from_numpy(rng.standard_normal((1, h, d))).bfloat16() for h in (hkv, hkv, 8)]
        for dst, src in zip((k, v, q), rows):
            dst.copy_(src)
        start.fill_(60 + i)
        ctx.fill_(61 + i)
        graph.replay()
        O.append(pool, L, table, [60 + i], [0, 1], rows[0].double().numpy(), rows[1].double().numpy())
        assert np.array_equal(g.data.cpu().numpy(), pool)
        check_decode(L, table, pool, [61 + i], rows[2].double().numpy(), 0.1, out)
    assert int(err) == 0 and jf.workspace_status(ws) == 0


# --------------------------------------------------------------------------
# chunks, page copies, refusals
# --------------------------------------------------------------------------
def prefill_bound(ref, mass, n, top, q, k, scale):
    """out_bound, with q times scale entering as fp16 (2^-12 of each product, so a weight is off by at most twice
    2^-11 of its largest sum of |q k|), and weights that enter at 2^-14 of the largest with 2^-25 of it."""
    d = 2.0 ** -11 * (np.abs(q) @ np.abs(k).T * abs(scale)).max(-1)[:, None]
    return C.out_bound(ref, mass, n, top) + mass * 2 * d + n * top * 448 * 2.0 ** -25


@pytest.mark.parametrize("hq,hkv,d,p,start,count,splits,causal", [
    (24, 4, 256, 256, [0], [1], 1, True),
    (24, 4, 256, 64, [500], [129], 1, True),
    (8, 2, 128, 128, [31, 0, 700], [65, 64, 1], 1, True),
    (8, 2, 128, 64, [0, 333], [200, 50], 3, True),
    (6, 1, 256, 128, [1000, 5], [7, 0], 4, True),
    (2, 2, 128, 256, [100], [300], 1, False),
    (16, 1, 128, 64, [63], [2], 1, True),
])
@pytest.mark.parametrize("spread", [0, 12])
def test_prefill(hq, hkv, d, p, start, count, splits, causal, spread):
    rng = np.random.default_rng(hq * d + sum(start) + spread)
    ctx = [s + c for s, c in zip(start, count)]
    L = O.Layout(hkv, p, d)
    table, pages = C.tables(rng, [-(-n // p) for n in ctx])
    pool = O.new_pool(L, pages, 0xFF)
    off = np.concatenate([[0], np.cumsum(ctx)])
    n = int(off[-1])
    O.append(pool, L, table, [0] * len(ctx), off, C.rows(rng, n, hkv, d), C.rows(rng, n, hkv, d, spread))
    g = C.gpu_pool(L, pool)
    q = torch.from_numpy(rng.standard_normal((sum(count), hq, d))).bfloat16().double().numpy()
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    scale = float(np.float32(1 / math.sqrt(d)))
    if len(ctx) == 1 and splits == 1:
        ws = torch.full((256,), 0, dtype=torch.uint8, device=DEV)
        jf.jf_prefill_chunk_attn(g, C.ints(table)[0], C.bf16(q), start[0], scale, causal, out, ws)
    else:
        ws = jf.prefill_batch_workspace(sum(count), hq, d, splits, format=jf.JF_FMT_E4M3_B32)
        ws[256:] = 0xFF
        jf.jf_prefill_batch_attn(g, C.ints(table), start, count, C.bf16(q), scale, causal, out, ws, splits)
    assert jf.workspace_status(ws) == 0
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    r = 0
    G = hq // hkv
    for b, (s, c) in enumerate(zip(start, count)):
        if c == 0:
            continue
        k, v = O.read(pool, L, table[b], ctx[b])
        mine = q[r:r + c]
        limit = s + 1 + np.arange(c) if causal else None
        ref, w, mass = O.attend(k, v, mine, scale, limit)
        for h in range(hq):
            top = (w[:, h].max(0)[:, None] * np.abs(v[:, h // G])).max(initial=0)
            bound = prefill_bound(ref[:, h], mass[:, h], ctx[b], top if spread == 0 else mass[:, h].max(-1)[:, None],
                                  mine[:, h], k[:, h // G], scale)
            err = np.abs(got[r:r + c, h] - ref[:, h])
            assert (err <= bound).all(), (b, h, float((err - bound).max()))
        r += c


def test_prefill_wave_balanced_equals_one_launch():
    """A chunk whose tail splits its history: within rounding of the single launch."""
    rng = np.random.default_rng(31)
    hkv, d, p, start, c, hq = 4, 128, 256, 9000, 2000, 24
    L = O.Layout(hkv, p, d)
    pages = -(-(start + c) // p)
    g = jf.KVPool.allocate(pages, p, hkv, d, format=jf.JF_FMT_E4M3_B32)
    table = C.ints(rng.permutation(pages)[None])
    x = [torch.randn(start + c, hkv, d, device=DEV).bfloat16() for _ in range(2)]
    err = gpu_append(g, table.cpu().numpy(), [0], [0, start + c], *x)
    q = torch.randn(c, hq, d, device=DEV).bfloat16()
    big = jf.prefill_chunk_workspace(g, start, c, hq)
    assert big.numel() > 256
    outs = []
    for ws in (big, torch.zeros(256, dtype=torch.uint8, device=DEV)):
        out = torch.full_like(q, float("nan"))
        jf.jf_prefill_chunk_attn(g, table[0], q, start, 1 / math.sqrt(d), True, out, ws)
        assert jf.workspace_status(ws) == 0
        outs.append(out.float())
    assert int(err) == 0
    # both round to bf16 what differs by the order of fp32 sums and by P's fp16 rounding (below 2^-10 of the mass)
    assert (outs[0] - outs[1]).abs().max() <= 2.0 ** -7 * outs[1].abs().max()


@pytest.mark.parametrize("hq,hkv,d,p,start,c,causal", [
    (24, 4, 256, 256, 3400, 840, True),      # 80 pairs: 4 left over, their histories in many parts
    (24, 4, 256, 64, 7001, 1700, False),     # 164 pairs: 12 left over
    (12, 3, 128, 128, 9000, 2005, True),     # odd lengths, 96 pairs: 21 left over
    (7, 1, 128, 64, 13001, 3001, True),      # 7 query heads: 84 pairs, padding rows
    (4, 4, 256, 128, 16400, 4100, True),     # one query head a KV head: 68 pairs, one wave
])
def test_prefill_divided_last_wave_equals_undivided(hq, hkv, d, p, start, c, causal):
    """Pairs beyond whole waves with their histories in parts: within rounding of the undivided launch."""
    rng = np.random.default_rng(c)
    pages = -(-(start + c) // p)
    g = jf.KVPool.allocate(pages, p, hkv, d, format=jf.JF_FMT_E4M3_B32)
    table = C.ints(rng.permutation(pages)[None])
    torch.manual_seed(c)
    x = [torch.randn(start + c, hkv, d, device=DEV).bfloat16() for _ in range(2)]
    err = gpu_append(g, table.cpu().numpy(), [0], [0, start + c], *x)
    q = torch.randn(c, hq, d, device=DEV).bfloat16()
    big = jf.prefill_chunk_workspace(g, start, c, hq)
    big[256:] = 0xFF                         # NaN: what no part writes is not read
    outs = []
    for ws in (big, big, torch.zeros(256, dtype=torch.uint8, device=DEV)):
        out = torch.full_like(q, float("nan"))
        jf.jf_prefill_chunk_attn(g, table[0], q, start, 1 / math.sqrt(d), causal, out, ws)
        assert jf.workspace_status(ws) == 0
        outs.append(out)
    assert int(err) == 0
    assert torch.equal(outs[0], outs[1])     # the same bits every time
    a, b = outs[0].double(), outs[2].double()
    assert torch.isfinite(a).all()
    # Each form rounds P to fp16 (2^-11 of it), sums in fp32 and rounds once to bf16 (2^-8):
    # together they differ by at most 2 (2^-11 max|v| + 2^-8 |out|) and a little for the sums.
    top = x[1].abs().max().double() * (1 + 2.0 ** -4)
    assert ((a - b).abs() <= 2 * (2.0 ** -11 + 2.0 ** -16) * top + 2 * 2.0 ** -8 * b.abs()).all()


@pytest.mark.parametrize("hq,d", [(8, 128), (6, 256), (2, 128)])
def test_decode_weights_of_a_page_outside_the_pool(hq, d):
    """Positions of a bad page draw no weight (whatever the workspace held), and a request of bad pages alone gives
    zeros; the others' weights and outputs are those of a context without them."""
    rng = np.random.default_rng(hq)
    hkv, p, ctx = 2, 64, [200, 130, 64]
    L, table, pool = C.filled(rng, hkv, p, d, ctx)
    g = C.gpu_pool(L, pool)
    q = torch.randn(3, hq, d, device=DEV).bfloat16()
    bad = table.copy()
    bad[0, 1], bad[1, :3], bad[2, 0] = len(pool), -1, 1 << 30
    w_in = torch.rand(3, hkv, 200, device=DEV)

    def run(tbl, splits):
        out, w = torch.full_like(q, float("nan")), torch.full_like(w_in, float("nan"))
        ws = jf.decode_weights_workspace(3, hq, hkv, d, splits, 200)
        ws[256:] = 0xFF                              # NaN partials and scores
        jf.jf_paged_decode_weights_attn(g, C.ints(tbl), C.ints(ctx), q, 0.1, out, w_in, w, ws, splits)
        return out, w, jf.workspace_status(ws)

    for splits in (1, 4):
        out, w, status = run(bad, splits)
        assert status == jf.binding.JF_DEV_ERR_PAGE_ID
        assert (out[1:] == 0).all()
        for b in (1, 2):
            assert torch.equal(w[b, :, :ctx[b]], w_in[b, :, :ctx[b]])
        assert torch.equal(w[0, :, 64:128], w_in[0, :, 64:128])
        # request 0 without its second page: positions 0..63 and 128..199
        k, v = O.read(pool, L, table[0], 200)
        seen = np.r_[0:64, 128:200]
        ref, pr, mass = O.attend(k[seen], v[seen], q[:1].double().cpu().numpy(), float(np.float32(0.1)))
        e = np.abs(out[0].double().cpu().numpy() - ref[0])
        assert (e <= C.out_bound(ref[0], mass[0], 200, np.abs(v).max())).all()
        got = (w[0].double() - w_in[0].double()).cpu().numpy()[:, seen]
        want = pr[0].reshape(hkv, hq // hkv, len(seen)).sum(1)
        # sums of up to 4 weights, each good to 2^-10 of itself, added in fp32 to a weight below 1
        assert (np.abs(got - want) <= 2.0 ** -10 * want + 2.0 ** -21).all()


def test_prefill_reports_a_page_outside_the_pool():
    """One request's bad page id is flagged; the other request's output does not change."""
    rng = np.random.default_rng(33)
    hq, hkv, d, p, start, count = 8, 2, 128, 64, [300, 200], [40, 24]
    ctx = [s + c for s, c in zip(start, count)]
    L, table, pool = C.filled(rng, hkv, p, d, ctx)
    g = C.gpu_pool(L, pool)
    q = torch.randn(sum(count), hq, d, device=DEV).bfloat16()

    def run(tbl, splits):
        out = torch.full_like(q, float("nan"))
        ws = jf.prefill_batch_workspace(sum(count), hq, d, splits, format=jf.JF_FMT_E4M3_B32)
        jf.jf_prefill_batch_attn(g, C.ints(tbl), start, count, q, 0.1, True, out, ws, splits)
        return out, jf.workspace_status(ws)

    for splits in (1, 3):
        good, status = run(table, splits)
        assert status == 0
        for bad in (-1, len(pool), 1 << 30, -(1 << 31)):
            t = table.copy()
            t[0, 2] = bad
            out, status = run(t, splits)
            assert status == jf.binding.JF_DEV_ERR_PAGE_ID
            assert torch.equal(out[count[0]:], good[count[0]:])


def test_positions_past_31_bits_are_refused():
    """A run that would end past the last 32-bit position does not fit, however long the page table is; runs that
    end at it do."""
    hkv, d, p = 1, 128, 256
    pages = 2
    g = jf.KVPool.allocate(pages, p, hkv, d, format=jf.JF_FMT_E4M3_B32)
    long = torch.zeros(1, (1 << 31) // p + 1, dtype=torch.int32, device=DEV)    # every entry page 0
    x = torch.randn(20, hkv, d, device=DEV).bfloat16()
    y, z = torch.full_like(x, -3.0), torch.full_like(x, -3.0)
    bit = jf.binding.JF_DEV_ERR_POSITION
    for start, fits in (((1 << 31) - 10, False), ((1 << 31) - 20, False), ((1 << 31) - 21, True)):
        before, err = g.data.clone(), flag()
        jf.jf_kv8_append(g, long, C.ints([start]), C.ints([0, 20]), x, x, err)
        assert int(err) == (0 if fits else bit) and torch.equal(g.data, before) == (not fits)
        err = flag()
        jf.jf_kv8_read(g, long, C.ints([start]), C.ints([0, 20]), y, z, err)
        assert int(err) == (0 if fits else bit)
        if not fits:
            assert (y == -3).all() and (z == -3).all()
    assert torch.equal(y, z) and (y.double() - x.double()).abs().max() <= 2.0 ** -4 * x.abs().max()


def test_checkpoint_and_restore_copy_the_pages():
    rng = np.random.default_rng(32)
    L, table, pool = C.filled(rng, 2, 64, 128, [150], fill=0x33)
    g = C.gpu_pool(L, pool)
    blob, err = torch.zeros(3 * L.page_bytes, dtype=torch.uint8, device=DEV), flag()
    jf.jf_kv_checkpoint(g, C.ints(table)[0], 3, blob, err)
    other = jf.KVPool.allocate(5, 64, 2, 128, format=jf.JF_FMT_E4M3_B32)
    jf.jf_kv_restore(other, C.ints([4, 0, 2]), 3, blob, err)
    assert int(err) == 0
    assert np.array_equal(other.data[[4, 0, 2]].cpu().numpy(), pool[table[0]])


def test_other_formats_and_entry_points_refuse():
    rng = np.random.default_rng(33)
    L, table, pool = C.filled(rng, 1, 64, 128, [10])
    g = C.gpu_pool(L, pool)
    four = jf.KVPool.allocate(1, 64, 1, 128)
    B = jf.binding
    x = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device=DEV)
    q, out = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 4, 128, dtype=torch.bfloat16, device=DEV)
    t, one, off = C.ints(table), C.ints([1]), C.ints([0, 1])
    ws = jf.decode_workspace(1, 4, 1, 128, 2)

    def refused(status, fn, *args):
        with pytest.raises(jf.JfError) as e:
            fn(*args)
        assert e.value.status == status
    U, I = B.JF_ERR_UNSUPPORTED, B.JF_ERR_INVALID_ARG
    refused(U, jf.jf_kv8_append, four, t, one, off, x, x)
    refused(U, jf.jf_kv8_read, four, t, one, off, x, x)
    refused(U, jf.jf_kv_quantize_append, g, t, C.ints([0]), C.ints([0]), x, x)
    refused(U, jf.jf_paged_verify_attn, g, t, one, q[:, None], 0.1, out[:, None], ws, 2)
    refused(U, jf.jf_paged_decode_append_attn, g, t, one, x, x, q, 0.1, out, ws, 2)
    refused(U, jf.jf_paged_decode_attn_noalloc, g, t, one, q, 0.1, out, 2)
    w = torch.zeros(1, 1, 16, device=DEV)
    wws = jf.decode_weights_workspace(1, 4, 1, 128, 2, 16)
    refused(U, jf.jf_paged_decode_weights_attn, four, t, one, q, 0.1, out, None, w, wws, 2)
    refused(B.JF_ERR_WORKSPACE_TOO_SMALL, jf.jf_paged_decode_weights_attn, g, t, one, q, 0.1, out, None, w, ws, 2)
    refused(B.JF_ERR_WORKSPACE_TOO_SMALL, jf.jf_paged_decode_attn, g, t, one, q, 0.1, out, ws[:512], 2)
    refused(I, jf.jf_paged_decode_attn, g, t, one, q, float("nan"), out, ws, 2)
    q9 = torch.zeros(1, 9, 128, dtype=torch.bfloat16, device=DEV)
    refused(U, jf.jf_paged_decode_attn, g, t, one, q9, 0.1, torch.zeros_like(q9), jf.decode_workspace(1, 9, 1, 128, 2), 2)
    for bad in (dict(start=C.ints([1, 2])), dict(off=C.ints([0])), dict(x=x[:, :, :64])):
        with pytest.raises(ValueError):
            jf.jf_kv8_append(g, t, bad.get("start", one), bad.get("off", off), bad.get("x", x), x)
    with pytest.raises(TypeError):
        jf.jf_kv8_append(g, t, one, off, x.float(), x)
    with pytest.raises(ValueError):
        jf.KVPool.allocate(1, 48, 1, 128, format=jf.JF_FMT_E4M3_B32)
