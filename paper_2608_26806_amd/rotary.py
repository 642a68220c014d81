"""Rotary positions: what each pair of a head's values turns by at one position.

Pruned tokens keep the positions they had, of one plane or of several (running
position, row and column of an image's patches), so a rotation takes position
ids and not a running count.  ``rotary_frequencies`` gives the frequencies of
the pairs, stretched for contexts longer than those a model was trained on;
``Rotary`` keeps them on the device as the kernels take them.

    rotary = Rotary(128, *rotary_frequencies(128, 1e6, "parts", factor=8, trained=4096))
    q, k = A.norm_rotary(rotary, pos, q, k, q_weight=wq, k_weight=wk)
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import numpy as np
import torch

from . import avtp as A

PAIRS = ("half", "interleaved")
_TWO_PI = 2 * np.longdouble("3.14159265358979323846264338327950288")


def rotary_frequencies(rot_dim: int, base: float = 10000.0, stretch: Optional[str] = None, factor: float = 1.0,
                       trained: int = 0, fast: float = 32.0, slow: float = 1.0):
    """Frequencies (radians a position, float64 [rot_dim / 2]) and the scale of
    the rotated values: base^(-2 i / rot_dim), and by ``stretch``

    - ``"linear"``: all divided by ``factor`` (positions drawn together; position
      interpolation, arXiv:2306.15595);
    - ``"base"``: from base * factor^(rot_dim / (rot_dim - 2)), so that the slowest
      pair is divided by ``factor`` and the fastest stays ("NTK-aware", described in
      arXiv:2309.00071);
    - ``"parts"``: pairs that make ``fast`` turns or more within ``trained``
      positions stay, those that make ``slow`` or fewer are divided by
      ``factor``, linearly in the pair's number between (the borders moved outwards to
      whole pairs, the first of which always stays); values scaled by 0.1 ln(factor) + 1
      (YaRN, arXiv:2309.00071, its ramp taken over the pairs);
    - ``"wavelength"``: the same borders, linearly in the number of turns, not scaled
      ("NTK-by-parts" of the same paper).
    """
    if rot_dim < 4 or rot_dim % 2 or not base > 0 or not factor >= 1:
        raise ValueError("an even rot_dim of 4 or more, a positive base and a factor of 1 or more are needed")
    i = np.arange(rot_dim // 2, dtype=np.float64)
    if stretch == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-2 * i / rot_dim)
    if stretch in (None, "base"):
        return f, 1.0
    if stretch == "linear":
        return f / factor, 1.0
    if stretch not in ("parts", "wavelength"):
        raise ValueError(f"stretch: {stretch!r}")
    if trained < 1 or not fast > slow > 0:
        raise ValueError("trained positions and fast > slow > 0 turns are needed")
    if stretch == "wavelength":
        stay = np.clip((trained * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
        return f * stay + f / factor * (1 - stay), 1.0
    pair = lambda turns: rot_dim * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    first, last = max(0, math.floor(pair(fast))), min(rot_dim - 1, math.ceil(pair(slow)))
    stay = 1 - np.clip((i - first) / max(last - first, 0.001), 0, 1)  # (both borders on one pair: a step)
    return f * stay + f / factor * (1 - stay), 0.1 * math.log(factor) + 1


class Rotary:
    """The rotation of the first ``rot_dim`` values of a head, by ``freqs``
    (radians a position; base^(-2 i / rot_dim) if none are given).

    ``pairs``: "half" turns values (i, i + rot_dim / 2), "interleaved" (2 i, 2 i + 1).
    ``planes``: for each pair the plane of positions that turns it (the first
    for all if none are given).  Rotated values are multiplied by ``scale``.
    The inverse rotation has negated frequencies."""

    def __init__(self, rot_dim: int, freqs: Optional[Sequence[float]] = None, scale: float = 1.0,
                 base: float = 10000.0, pairs: str = "half", planes: Optional[Sequence[int]] = None,
                 device="cuda"):
        if pairs not in PAIRS:
            raise ValueError(f"pairs: one of {PAIRS} is needed, got {pairs!r}")
        if rot_dim < 16 or rot_dim % 16:
            raise ValueError(f"rot_dim: a multiple of 16 is needed, got {rot_dim}")
        if freqs is None:
            freqs = rotary_frequencies(rot_dim, base)[0]
        f = np.asarray(freqs, dtype=np.float64)
        if f.shape != (rot_dim // 2,) or not np.isfinite(f).all():
            raise ValueError(f"freqs: {rot_dim // 2} finite numbers are needed")
        if planes is not None:
            planes = [int(p) for p in planes]
            if len(planes) != rot_dim // 2 or min(planes) < 0 or max(planes) >= A.MAX_PLANES:
                raise ValueError(f"planes: {rot_dim // 2} numbers below {A.MAX_PLANES} are needed")
        # fractions of a turn in 64 bits; whole turns drop out (the long double's 64-bit
        # mantissa holds each to 2^-64 of itself)
        x = f.astype(np.longdouble) / _TWO_PI
        turns = np.rint(np.ldexp(x - np.floor(x), 64))
        turns = np.where(turns < np.ldexp(np.longdouble(1), 64), turns, 0).astype(np.uint64)
        self.rot_dim, self.pairs, self.scale = rot_dim, pairs, float(scale)
        self.n_planes = 1 if planes is None else max(planes) + 1
        self.turns = torch.from_numpy(turns.view(np.int64)).to(device)
        self.planes = None if planes is None or self.n_planes == 1 else \
            torch.tensor(planes, dtype=torch.int32, device=device)
        self.st = A._Rotary(self.turns.data_ptr(), None if self.planes is None else self.planes.data_ptr(), rot_dim,
                            PAIRS.index(pairs), self.n_planes, self.scale)

    def ref(self):
        A._page_arg(self.turns, "rotary", self.rot_dim // 2, torch.int64)
        A._page_arg(self.planes, "rotary", self.rot_dim // 2)
        return ctypes.byref(self.st)
