"""fp64 definition of rotary positions with several axes."""
import numpy as np


def axes_of(sections, layout):
    half, n = sum(sections), len(sections)
    if layout == "sectioned":
        return [a for a, m in enumerate(sections) for _ in range(m)]
    return [i % n if i < n * sections[i % n] else 0 for i in range(half)]


def rotate(x, pos, axis, inv_freq, pairing, inverse=False):
    """x fp64 [tokens, heads, D], pos int [axes, tokens], inv_freq the fp32 frequencies."""
    half = len(axis)
    out = np.array(x, dtype=np.float64)
    for i in range(half):
        a, b = (i, i + half) if pairing == "half" else (2 * i, 2 * i + 1)
        p = pos[axis[i]].astype(np.longdouble) * np.longdouble(inv_freq[i])
        p = np.fmod(p, 2 * np.longdouble("3.14159265358979323846264338327950288"))
        c, s = np.cos(p).astype(np.float64)[:, None], np.sin(p).astype(np.float64)[:, None]
        s = -s if inverse else s
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., a] * s + x[..., b] * c
    return out
