"""Oracle: training on packed documents of long contexts, fp64: rotary positions
on a part of each head with scaled frequencies, forward and backward.

TEST INFRASTRUCTURE ONLY (see the package docstring).

  * Rotary part: r pairs of a head's columns from `offset` on, (i, i + r) or
    (2i, 2i + 1), turned by amplitude * rotation(position * w_i); w = base^(-i/r),
    interpolated (w / f), of a larger base (b f^(r / (r - 1)) for r pairs), or by
    parts: w (g + (1 - g) / f), g = the turns in the trained context, from `low`
    (0) to `high` (1).
"""
from __future__ import annotations

import numpy as np


def part_frequencies(rot, base, scaling="none", factor=1.0, low=0.0, high=1.0, original=1,
                     pair_factors=None):
    r = rot // 2
    i = np.arange(r)
    if scaling == "base":
        base = base * factor ** (r / (r - 1))
    w = float(base) ** (-i / r)
    if scaling == "linear":
        w = w / factor
    if scaling == "parts":
        turns = original * w / (2.0 * np.pi)
        g = np.clip((turns - low) / (high - low), 0.0, 1.0)
        w = w * g + w * (1.0 - g) / factor
    return w if pair_factors is None else w / np.asarray(pair_factors, np.float64)


def part_columns(rot, offset, interleaved):
    """(first, second) column of every pair."""
    i = np.arange(rot // 2)
    return (offset + 2 * i, offset + 2 * i + 1) if interleaved else (offset + i,
                                                                     offset + i + rot // 2)


def rope_part(x, positions, rot, offset, interleaved, w, amplitude=1.0, backward=False):
    """x [T, heads, d]; backward: the transposed matrix."""
    ang = positions[:, None] * w
    c, s = amplitude * np.cos(ang)[:, None], amplitude * np.sin(ang)[:, None]
    if backward:
        s = -s
    a, b = part_columns(rot, offset, interleaved)
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y
