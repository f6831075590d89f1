"""Oracle: an attention branch with LayerNorm, rotary positions with several
axes and sliding-window attention with sinks, forward and backward, fp64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

  * LayerNorm: y = (x - m) r g + b, m the row's mean, r = (mean((x - m)^2) +
    eps)^(-1/2).
  * Rotary axes: pair (i, i + d/2) of a head belongs to one axis and turns by
    that axis' position times the pair's frequency.
  * Window: key j is visible to query i of its batch row iff j <= i and
    (i - j < window or j < sinks), both below the row's length; a row behind
    the length has zero output, lse -inf and no gradient.
"""
from __future__ import annotations

import numpy as np


def layernorm_fwd(x, g, b, eps):
    """(y, mean, rstd); b may be None."""
    m = x.mean(axis=1)
    r = 1.0 / np.sqrt(((x - m[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - m[:, None]) * r[:, None] * g
    return (y if b is None else y + b), m, r


def layernorm_bwd(x, g, m, r, dy):
    """(dx, dg, db) of y = xh g + b with xh = (x - m) r."""
    xh = (x - m[:, None]) * r[:, None]
    u = dy * g
    dx = r[:, None] * (u - u.mean(axis=1, keepdims=True)
                       - xh * (u * xh).mean(axis=1, keepdims=True))
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


def pair_axes(pairs, interleaved):
    """[(axis, index within the axis)] of every pair: sections in axis order, or
    dealt in turn, an axis that has its share being passed over."""
    if not interleaved:
        return [(a, l) for a, n in enumerate(pairs) for l in range(n)]
    left, out = list(pairs), []
    while any(left):
        for a in range(len(pairs)):
            if left[a]:
                out.append((a, pairs[a] - left[a]))
                left[a] -= 1
    return out


def axes_frequencies(pairs, interleaved, own_ladder, base):
    half = sum(pairs)
    return np.array([base ** (-l / pairs[a] if own_ladder else -i / half)
                     for i, (a, l) in enumerate(pair_axes(pairs, interleaved))])


def rope_axes(x, positions, pairs, interleaved, own_ladder, base, inverse=False):
    """x [T, heads, d] rotated by positions [axes, T]; inverse: rotated back."""
    half = sum(pairs)
    axis = [a for a, _ in pair_axes(pairs, interleaved)]
    ang = positions[axis].T * axes_frequencies(pairs, interleaved, own_ladder, base)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None] * (-1.0 if inverse else 1.0)
    x1, x2 = x[..., :half], x[..., half:]
    return np.concatenate([x1 * c - x2 * s, x2 * c + x1 * s], axis=-1)


def visible(n, window, sinks):
    """[n, n] of bool: row i, key j."""
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    return (j <= i) & ((i - j < window) | (j < sinks))


def _probs(q, k, window, sinks):
    s = np.where(visible(len(q), window, sinks), (q @ k.T) / np.sqrt(q.shape[1]), -np.inf)
    top = s.max(axis=1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(axis=1, keepdims=True)
    return e / total, (top + np.log(total))[:, 0]


def window_attention(q, k, v, do, batch, seq, window, sinks, lens=None):
    """q, do [T, n_h, d], k, v [T, n_kv, d] (do may be None) -> dict of o, lse and,
    with do, dq, dk, dv; with each output but lse, under "err_" + its name, how
    far roundings to bf16 may move every element: of the probabilities and the
    score gradient, the operands of the products (2^-8 of each value), of o (as
    the backward reads it, in delta = sum do o), and of the output itself."""
    half = 2.0 ** -8
    nh, nkv, d = q.shape[1], k.shape[1], q.shape[2]
    names = ("o",) if do is None else ("o", "dq", "dk", "dv")
    like = dict(o=q, dq=q, dk=k, dv=v)
    r = {n: np.zeros_like(like[n]) for n in names}
    r.update({"err_" + n: np.zeros_like(like[n]) for n in names})
    r["lse"] = np.full((batch, nh, seq), -np.inf)
    for b in range(batch):
        n = seq if lens is None else min(max(int(lens[b]), 0), seq)
        rows = slice(b * seq, b * seq + n)
        for h in range(nh if n else 0):
            m = h // (nh // nkv)
            qh, kh, vh = q[rows, h], k[rows, m], v[rows, m]
            p, r["lse"][b, h, :n] = _probs(qh, kh, window, sinks)
            o = p @ vh
            r["o"][rows, h] = o
            err_o = half * (p @ np.abs(vh))
            r["err_o"][rows, h] = err_o
            if do is None:
                continue
            g = do[rows, h]
            r["dv"][rows, m] += p.T @ g
            r["err_dv"][rows, m] += half * (p.T @ np.abs(g))
            ds = p * (g @ vh.T - (g * o).sum(axis=1, keepdims=True))
            err_delta = (np.abs(g) * (err_o + half * np.abs(o))).sum(axis=1, keepdims=True)
            err_ds = half * np.abs(ds) + p * err_delta
            r["dq"][rows, h] = ds @ kh / np.sqrt(d)
            r["err_dq"][rows, h] = err_ds @ np.abs(kh) / np.sqrt(d)
            r["dk"][rows, m] += ds.T @ qh / np.sqrt(d)
            r["err_dk"][rows, m] += err_ds.T @ np.abs(qh) / np.sqrt(d)
    for n in names:
        r["err_" + n] += half * np.abs(r[n])
    return r
