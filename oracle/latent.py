"""Latent attention in fp64: the plain definitions on dense rows, and the paged pool's addressing.

A position is one row of R latent and 64 rotated key channels; a page is P rows.
"""
import numpy as np

ROT = 64


def gather(pool, table_row, n):
    """Positions 0 .. n - 1 of a request: pool [pages, P, R + 64] -> [n, R + 64]."""
    P = pool.shape[1]
    t = np.arange(n)
    return pool[np.asarray(table_row)[t // P], t % P] if n else np.zeros((0, pool.shape[2]))


def softmax(x):
    """Rows of x over the last axis; -inf leaves a position out."""
    w = np.exp(x - x.max(-1, keepdims=True))
    return w / w.sum(-1, keepdims=True)


def decode(q, kv, scale):
    """q [H, R + 64] over kv [n, R + 64] -> out [H, R], and sum of |weight x latent| (zeros where n is 0)."""
    R = kv.shape[1] - ROT
    if len(kv) == 0:
        return np.zeros((len(q), R)), np.zeros((len(q), R))
    w = softmax(scale * (q @ kv.T))
    return w @ kv[:, :R], w @ np.abs(kv[:, :R])


def expand(kv, w_k, w_v):
    """Keys [n, 192] and values [n, 128] of one head."""
    R = kv.shape[1] - ROT
    return np.concatenate([kv[:, :R] @ w_k.T, kv[:, R:]], 1), kv[:, :R] @ w_v.T


def prefill(q, kv, q_start, w_k, w_v, scale, causal):
    """q [C, H, 192] -> out [C, H, 128], sum of |weight x value|, and the largest over a row's positions of the sum of
    |q x key| (what a relative rounding of keys may move a score by)."""
    C, H, _ = q.shape
    n = len(kv)
    out, mass, reach = np.zeros((C, H, 128)), np.zeros((C, H, 128)), np.zeros((C, H))
    seen = (np.arange(n) <= q_start + np.arange(C)[:, None]) if causal else np.ones((C, n), bool)
    for h in range(H):
        k, v = expand(kv, w_k[h], w_v[h])
        x = np.where(seen, scale * (q[:, h] @ k.T), -np.inf)
        w = softmax(x)
        out[:, h], mass[:, h] = w @ v, w @ np.abs(v)
        reach[:, h] = (np.where(seen, np.abs(q[:, h]) @ np.abs(k).T, 0)).max(1)
    return out, mass, reach
