"""Pins of oracle.branch: finite differences of every backward, and closed forms
that a plausible mistake breaks (LayerNorm's invariances, a rotation's norm and
its dependence on position differences, the window against full attention and
against one row worked out by hand)."""
import numpy as np
import pytest

from oracle import branch, dense
from fdcheck import central_diff, sample_indices, rel_err


def test_layernorm_backward_finite_differences():
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((5, 16)) + 0.7, rng.standard_normal((5, 16))
    g, b = 1.0 + 0.3 * rng.standard_normal(16), rng.standard_normal(16)

    def f():
        return float((branch.layernorm_fwd(x, g, b, 1e-3)[0] * dy).sum())
    _, m, r = branch.layernorm_fwd(x, g, b, 1e-3)
    for got, wrt in zip(branch.layernorm_bwd(x, g, m, r, dy), (x, g, b)):
        idx = np.arange(wrt.size)
        assert rel_err(got.ravel(), central_diff(f, wrt, idx)) <= 1e-6


def test_layernorm_ignores_a_row_s_offset_and_scale():
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((4, 32)), rng.standard_normal(32)
    y, _, _ = branch.layernorm_fwd(x, g, None, 0.0)
    moved, m, _ = branch.layernorm_fwd(3.0 * x + 5.0, g, None, 0.0)
    assert np.allclose(y, moved, rtol=0, atol=1e-12)
    assert np.allclose(m, 3.0 * x.mean(axis=1) + 5.0)
    assert np.allclose(((y / g) ** 2).mean(axis=1), 1.0)


def test_pairs_of_axes():
    assert branch.pair_axes([2, 3], False) == [(0, 0), (0, 1), (1, 0), (1, 1), (1, 2)]
    assert branch.pair_axes([3, 1, 2], True) == [(0, 0), (1, 0), (2, 0), (0, 1), (2, 1), (0, 2)]


@pytest.mark.parametrize("pairs,inter,own", [([4, 6, 6], False, False), ([6, 5, 5], True, False),
                                             ([8, 8], False, True), ([3, 13], True, True)])
def test_rope_axes_is_a_rotation_of_position_differences(pairs, inter, own):
    rng = np.random.default_rng(3)
    n, d, T = len(pairs), 2 * sum(pairs), 6
    pos = rng.integers(0, 50, (n, T))
    q, k = rng.standard_normal((T, 2, d)), rng.standard_normal((T, 2, d))

    def turn(x, p, inverse=False):
        return branch.rope_axes(x, p, pairs, inter, own, 100.0, inverse)
    y = turn(q, pos)
    assert np.allclose((y ** 2).sum(-1), (q ** 2).sum(-1))
    assert np.allclose(turn(y, pos, True), q)
    shift = rng.integers(0, 9, (n, 1))
    same = np.einsum("thd,shd->hts", turn(q, pos), turn(k, pos))
    moved = np.einsum("thd,shd->hts", turn(q, pos + shift), turn(k, pos + shift))
    assert np.allclose(same, moved)
    # an axis' position turns that axis' pairs alone
    other = pos.copy()
    other[0] += 7
    changed = np.abs(turn(q, other) - y).max(axis=(0, 1)) > 1e-9
    mine = np.array([a == 0 for a, _ in branch.pair_axes(pairs, inter)] * 2)
    assert np.array_equal(changed, mine)


def test_rope_axes_of_equal_positions_is_plain_rope():
    rng = np.random.default_rng(4)
    x, pos = rng.standard_normal((7, 3, 32)), np.arange(7) * 5
    plain = dense.rope_fwd(x, 1, 7, 1e4, pos)
    for inter in (False, True):
        y = branch.rope_axes(x, np.stack([pos] * 3), [4, 6, 6], inter, False, 1e4)
        assert np.allclose(y, plain)


def test_window_of_the_whole_row_is_causal_attention():
    rng = np.random.default_rng(5)
    B, S, nh, nkv, d = 2, 9, 4, 2, 8
    q, do = rng.standard_normal((B * S, nh, d)), rng.standard_normal((B * S, nh, d))
    k, v = rng.standard_normal((B * S, nkv, d)), rng.standard_normal((B * S, nkv, d))
    o, lse = dense.attention_fwd(q, k, v, B, S)
    for window, sinks in ((9, 0), (100, 3), (1, 9)):
        r = branch.window_attention(q, k, v, do, B, S, window, sinks)
        assert np.allclose(r["o"], o) and np.allclose(r["lse"], lse)
        for got, ref in zip((r["dq"], r["dk"], r["dv"]), dense.attention_bwd(q, k, v, do, B, S)):
            assert np.allclose(got, ref)


def test_visible_keys_of_one_row():
    vis = branch.visible(10, 3, 2)
    assert np.flatnonzero(vis[7]).tolist() == [0, 1, 5, 6, 7]
    assert np.flatnonzero(vis[3]).tolist() == [0, 1, 2, 3]
    assert np.flatnonzero(vis[0]).tolist() == [0]
    assert branch.visible(6, 1, 0).sum() == 6


@pytest.mark.parametrize("window,sinks,lens", [(3, 0, None), (2, 2, None), (4, 1, (7, 0, 5))])
def test_window_attention_backward_finite_differences(window, sinks, lens):
    rng = np.random.default_rng(6)
    B, S, nh, nkv, d = 3, 7, 2, 1, 4
    q, do = rng.standard_normal((B * S, nh, d)), rng.standard_normal((B * S, nh, d))
    k, v = rng.standard_normal((B * S, nkv, d)), rng.standard_normal((B * S, nkv, d))

    def f():
        return float((branch.window_attention(q, k, v, None, B, S, window, sinks, lens)["o"]
                      * do).sum())
    r = branch.window_attention(q, k, v, do, B, S, window, sinks, lens)
    for got, wrt in ((r["dq"], q), (r["dk"], k), (r["dv"], v)):
        idx = sample_indices(wrt.size, 90, rng)
        assert rel_err(got.ravel()[idx], central_diff(f, wrt, idx)) <= 1e-6
    for b in range(B):
        n = S if lens is None else lens[b]
        pad = slice(b * S + n, (b + 1) * S)
        assert not r["o"][pad].any() and not r["dq"][pad].any() and not r["dv"][pad].any()
        assert np.all(np.isneginf(r["lse"][b, :, n:])) and np.all(np.isfinite(r["lse"][b, :, :n]))
