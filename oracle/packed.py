"""Oracle: training on packed documents of long contexts, fp64: rotary positions
on a part of each head with scaled frequencies and attention over packed sequences,
forward and backward, and AdamW with moments of 8 bits.

TEST INFRASTRUCTURE ONLY (see the package docstring).

  * Rotary part: r pairs of a head's columns from `offset` on, (i, i + r) or
    (2i, 2i + 1), turned by amplitude * rotation(position * w_i); w = base^(-i/r),
    interpolated (w / f), of a larger base (b f^(r / (r - 1)) for r pairs), or by
    parts: w (g + (1 - g) / f), g = the turns in the trained context, from `low`
    (0) to `high` (1).
  * Packed attention: every sequence a row of its own, causal, with or without a
    window; offsets are taken as their running maximum cut to [0, tokens], of a
    sequence longer than max_seq the first max_seq rows.
  * Moments of 8 bits: blocks of 256 share their largest magnitude s; m's code q
    stands for q |q| s / 127^2, v's for (q / 255)^4 s; a value between those of two
    codes takes the upper one iff u (upper - lower) < value - lower, u in (0, 1)
    drawn from (seed, tensor, element) by a 32-bit hash. Codes are decided by fp32
    operations rounded one by one, so these are computed in float32 here.
"""
from __future__ import annotations

import numpy as np

from . import branch


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


BLOCK = 256
F32 = np.float32


def _mix(x):
    x = np.asarray(x, np.uint64) & 0xFFFFFFFF
    x = ((x ^ (x >> 16)) * 0xE699D49D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xC570DA33) & 0xFFFFFFFF
    return x ^ (x >> 16)


def moment_draws(n, tensor, seed):
    """(u of m, u of v) fp32 [n]; seed None: halves (to the nearest)."""
    if seed is None:
        return np.full(n, F32(0.5)), np.full(n, F32(0.5))
    r = _mix(np.arange(n, dtype=np.uint64) ^ _mix(_mix(seed) + np.uint64(tensor)))
    return (((r & 0xFFFF).astype(F32) + F32(0.5)) * F32(2.0 ** -16),
            ((r >> 16).astype(F32) + F32(0.5)) * F32(2.0 ** -16))


def _blocks(x):
    n = -(-x.size // BLOCK) * BLOCK
    return np.concatenate([x, np.zeros(n - x.size, x.dtype)]).reshape(-1, BLOCK)


def _scales(x):
    top = np.abs(_blocks(x)).max(axis=1)
    return np.where(top < F32(2.0 ** -94), F32(0), top).astype(F32)


def _spread(s, n):
    return np.repeat(s, BLOCK)[:n]


def decode_m(q, s):
    q = q.astype(np.int32)
    return (q * np.abs(q)).astype(F32) * _spread(s * F32(1 / 16129), q.size)


def decode_v(q, s):
    q = q.astype(np.int32)
    c = (q * q).astype(F32) * F32(1 / 65025)
    return (c * c) * _spread(s, q.size)


def _inverse(s, top):
    return F32(top) * np.divide(F32(1), s, out=np.zeros_like(s), where=s > 0)


def encode_m(m, u):
    s = _scales(m)
    a = np.abs(m) * _spread(_inverse(s, 16129.0), m.size)
    q = np.floor(np.sqrt(a))
    q = q + (u * (F32(2) * q + F32(1)) < a - q * q)
    return (np.minimum(q, 127) * np.sign(m)).astype(np.int8), s


def encode_v(v, u):
    s = _scales(v)
    x = v * _spread(_inverse(s, 255.0 ** 4), v.size)
    q = np.floor(np.sqrt(np.sqrt(x)))
    lo, hi = (q * q) * (q * q), ((q + F32(1)) * (q + F32(1))) * ((q + F32(1)) * (q + F32(1)))
    q = q + (u * (hi - lo) < x - lo)
    return np.where((v > 0) & (_spread(s, v.size) > 0), np.clip(q, 1, 255), 0).astype(np.uint8), s


def moments_step(g, qm, sm, qv, sv, beta1, beta2, clip):
    """The new moments fp32, before they are coded."""
    b1, b2, g = F32(beta1), F32(beta2), g.astype(F32) * F32(clip)
    m = decode_m(qm, sm) * b1 + (F32(1) - b1) * g
    return m, decode_v(qv, sv) * b2 + ((F32(1) - b2) * g) * g


def sequences(offsets, tokens, max_seq):
    """[(first row, rows)] of every sequence."""
    e = np.maximum.accumulate(np.clip(np.asarray(offsets, np.int64), 0, tokens))
    return [(int(a), min(int(b - a), max_seq)) for a, b in zip(e[:-1], e[1:])]


def covered(offsets, tokens, max_seq):
    """[tokens] of bool: rows of a sequence."""
    c = np.zeros(tokens, bool)
    for a, n in sequences(offsets, tokens, max_seq):
        c[a:a + n] = True
    return c


def positions(offsets, tokens, max_seq):
    p = np.full(tokens, -1, np.int64)
    for a, n in sequences(offsets, tokens, max_seq):
        p[a:a + n] = np.arange(n)
    return p


def attention(q, k, v, do, offsets, max_seq, window=0):
    """q, do [T, n_h, d], k, v [T, n_kv, d] (do may be None) -> dict of o, lse [n_h, T] and,
    with do, dq, dk, dv, each but lse with its "err_" as branch.window_attention's. Rows of
    no sequence are NaN."""
    T = len(q)
    names = ("o",) if do is None else ("o", "dq", "dk", "dv")
    like = dict(o=q, dq=q, dk=k, dv=v)
    r = {p + n: np.full_like(like[n], np.nan) for n in names for p in ("", "err_")}
    r["lse"] = np.full((q.shape[1], T), np.nan)
    for a, n in sequences(offsets, T, max_seq):
        if n == 0:
            continue
        s = slice(a, a + n)
        one = branch.window_attention(q[s], k[s], v[s], None if do is None else do[s], 1, n,
                                      window or n, 0)
        r["lse"][:, s] = one["lse"][0]
        for name in names:
            r[name][s], r["err_" + name][s] = one[name], one["err_" + name]
    return r
