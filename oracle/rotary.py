"""CPU oracle of the norm and rotation of heads: float64, a value at a time,
angles from whole numbers."""
from __future__ import annotations

import numpy as np


def angles(turns, pos):
    """Radians [n, pairs] of pos [pairs, n] times turns [pairs] / 2^64, whole turns
    taken away; exact but for the last rounding."""
    out = np.empty((len(pos[0]), len(turns)))
    for i, t in enumerate(turns):
        for n, p in enumerate(pos[i]):
            out[n, i] = 2 * np.pi * (int(t) * int(p) % (1 << 64) / 2.0 ** 64)
    return out


def norm_rotary(x, pos, turns, pairs, planes=None, scale=1.0, weight=None, eps=0.0):
    """x [n, heads, d], pos [planes, n] -> (rows, bound): what the roundings are
    relative to, |a| + |b| of a rotated pair, |y| of the other values."""
    x = np.asarray(x, dtype=np.float64)
    half = len(turns)
    y = x.copy()
    with np.errstate(all="ignore"):
        if weight is not None:
            y = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
        t = angles(turns, [pos[0 if planes is None else planes[i]] for i in range(half)])
        out, bound = y.copy(), np.abs(y)
        for i in range(half):
            a, b = (i, i + half) if pairs == "half" else (2 * i, 2 * i + 1)
            c, s = np.cos(t[:, i])[:, None], np.sin(t[:, i])[:, None]
            out[..., a] = scale * (y[..., a] * c - y[..., b] * s)
            out[..., b] = scale * (y[..., b] * c + y[..., a] * s)
            bound[..., a] = bound[..., b] = scale * (np.abs(y[..., a]) + np.abs(y[..., b]))
    return out, bound
