"""fp64 definition of the 8-bit block-scaled cache, its attention, and eviction by weight.

A code is an e4m3 value; positions 32 j .. 32 j + 31 of a KV head share a scale
2^e for K and one for V, e the smallest exponent with max|x| <= 448 * 2^e over
the finite values, limited to [-40, 40].  Page record: [K codes Hkv x P x D]
[V codes][K scales Hkv x P/32 fp32][V scales].
"""
import dataclasses
import math

import numpy as np

BLOCK, EMIN, EMAX, TOP = 32, -40, 40, 448.0


def _code_values():
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    x[(b & 127) == 127] = np.nan
    return np.where(b >= 128, -x, x)


VALUES = _code_values()
_POS = VALUES[:127]                       # 0 .. 448, rising


def round_codes(y: np.ndarray) -> np.ndarray:
    """e4m3 codes of fp64 values: nearest, ties to the even code, saturating; NaN -> 0x7f."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)      # first value >= a (the top one past it)
    lo = np.maximum(hi - 1, 0)
    up, down = _POS[hi] - a, a - _POS[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(a >= TOP, 126, c)
    c = np.where(np.signbit(y), c + 128, c)
    return np.where(np.isnan(y), 127, c).astype(np.uint8)


def exponent(x: np.ndarray) -> int:
    """The exponent that the values of one block call for."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    e = EMIN
    while e < EMAX and top > TOP * 2.0 ** e:
        e += 1
    return e


@dataclasses.dataclass(frozen=True)
class Layout:
    Hkv: int
    P: int
    D: int

    @property
    def page_bytes(self):
        return 2 * self.Hkv * (self.P * self.D + 4 * (self.P // BLOCK))

    def views(self, pool):
        """codes [pages, 2, Hkv, P, D] uint8 and scales [pages, 2, Hkv, P/32] fp32 of a pool."""
        n, at = len(pool), 2 * self.Hkv * self.P * self.D
        codes = pool[:, :at].reshape(n, 2, self.Hkv, self.P, self.D)
        scales = pool[:, at:].view(np.float32).reshape(n, 2, self.Hkv, self.P // BLOCK)
        return codes, scales


def new_pool(L: Layout, pages: int, fill: int = 0) -> np.ndarray:
    return np.full((pages, L.page_bytes), fill, dtype=np.uint8)


def _put(pool, L, page, kind, h, j, codes, e, first, last):
    at = 2 * L.Hkv * L.P * L.D
    row = ((kind * L.Hkv + h) * L.P + BLOCK * j) * L.D
    pool[page, row + first * L.D:row + last * L.D] = codes.reshape(-1)
    s = at + 4 * ((kind * L.Hkv + h) * (L.P // BLOCK) + j)
    pool[page, s:s + 4] = np.array([2.0 ** e], dtype=np.float32).view(np.uint8)


def append(pool, L: Layout, table, start, offsets, k, v):
    """k, v fp64 [rows, Hkv, D]."""
    for b, p0 in enumerate(start):
        rows = np.arange(offsets[b], offsets[b + 1])
        for blk in range(p0 // BLOCK, (p0 + len(rows) - 1) // BLOCK + 1 if len(rows) else 0):
            first, last = max(p0 - BLOCK * blk, 0), min(p0 + len(rows) - BLOCK * blk, BLOCK)
            page, j = table[b][BLOCK * blk // L.P], BLOCK * blk % L.P // BLOCK
            mine = rows[0] + BLOCK * blk + np.arange(first, last) - p0
            codes, scales = L.views(pool)
            for h in range(L.Hkv):
                for kind, x in enumerate((k, v)):
                    e = exponent(x[mine, h])
                    out = round_codes(x[mine, h] * 2.0 ** -e)
                    if first:
                        had = int(round(math.log2(scales[page, kind, h, j])))
                        if e > had:
                            old = VALUES[codes[page, kind, h, BLOCK * j:BLOCK * j + first]]
                            _put(pool, L, page, kind, h, j, round_codes(old * 2.0 ** (had - e)), e,
                                 0, first)
                        e = max(e, had)
                        out = round_codes(x[mine, h] * 2.0 ** -e)
                    _put(pool, L, page, kind, h, j, out, e, first, last)


def read(pool, L: Layout, row, n):
    """K and V [n, Hkv, D] fp64 of a request's first n positions; row: its pages."""
    codes, scales = L.views(pool)
    at = np.asarray(row)[:-(-n // L.P)].astype(np.int64)
    x = VALUES[codes[at]] * np.repeat(scales[at].astype(np.float64), BLOCK, -1)[..., None]
    x = x.transpose(1, 0, 3, 2, 4).reshape(2, -1, L.Hkv, L.D)[:, :n]
    return x[0], x[1]


def attend(k, v, q, scale, limit=None):
    """q [C, Hq, D] over k, v [n, Hkv, D]; limit[i]: positions query i sees (default all).
    Returns the output, the weights [C, Hq, n] and the sum of |weight * v|."""
    C, Hq, D = q.shape
    n, Hkv = k.shape[:2]
    G = Hq // Hkv
    out, mass = np.zeros((C, Hq, D)), np.zeros((C, Hq, D))
    w = np.zeros((C, Hq, n))
    for h in range(Hq):
        s = q[:, h] @ k[:, h // G].T * scale
        if limit is not None:
            s = np.where(np.arange(n)[None] < np.asarray(limit)[:, None], s, -np.inf)
        if n == 0:
            continue
        m = s.max(1, keepdims=True)
        p = np.exp(s - np.where(np.isinf(m), 0, m))
        l = p.sum(1, keepdims=True)
        w[:, h] = p / np.where(l > 0, l, 1)
        vh = v[:, h // G]
        out[:, h], mass[:, h] = w[:, h] @ vh, w[:, h] @ np.abs(vh)
    return out, w, mass


def keep(weights, budget, sinks, recent):
    """Positions kept of one row of weights, rising."""
    n = len(weights)
    w = np.where(np.isnan(weights), -np.inf, weights.astype(np.float64))
    nan = np.isnan(weights)
    t = np.arange(n)
    safe = (t < sinks) | (t >= n - recent)
    # protected, then by falling weight (NaN after -inf), then by rising position
    order = np.lexsort((t, nan, -w, ~safe))
    return np.sort(order[:min(n, budget)])


def evict(pool, L: Layout, table, ctx, weights, budget, sinks, recent, dst):
    """Compacts into dst's pages; returns kept and weights [B, Hkv, budget]."""
    B = len(ctx)
    kept = np.full((B, L.Hkv, budget), -1, dtype=np.int32)
    wout = np.zeros((B, L.Hkv, budget), dtype=np.float32)
    for b, n in enumerate(ctx):
        kv = read(pool, L, table[b], n)
        for h in range(L.Hkv):
            at = keep(weights[b, h, :n], budget, sinks, recent)
            kept[b, h, :len(at)] = at
            wout[b, h, :len(at)] = weights[b, h, at]
            for j0 in range(0, len(at), BLOCK):
                mine = at[j0:j0 + BLOCK]
                for kind in range(2):
                    x = kv[kind][mine, h]
                    e = exponent(x)
                    _put(pool, L, dst[b][j0 // L.P], kind, h, j0 % L.P // BLOCK,
                         round_codes(x * 2.0 ** -e), e, 0, len(mine))
    return kept, wout
