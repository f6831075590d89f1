"""Pins of oracle.packed: closed forms that a plausible mistake breaks, and finite
differences of every backward."""
import numpy as np
import pytest

from oracle import dense, packed
from fdcheck import central_diff, rel_err


# ----------------------------------------------------------- rotary part ----

PARTS = [(16, 0, False), (16, 0, True), (6, 4, False), (6, 10, True), (2, 14, False)]


@pytest.mark.parametrize("rot,offset,inter", PARTS)
def test_rope_part_turns_its_part_alone(rot, offset, inter):
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 16)), np.array([0, 3, 11, 4, 90])
    w = packed.part_frequencies(rot, 100.0)
    y = packed.rope_part(x, pos, rot, offset, inter, w)
    out = np.setdiff1d(np.arange(16), np.arange(offset, offset + rot))
    assert np.array_equal(y[..., out], x[..., out])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.array_equal(y[0], x[0])
    assert np.allclose(packed.rope_part(y, pos, rot, offset, inter, w, backward=True), x)
    # scores depend on position differences
    k = rng.standard_normal((5, 3, 16))
    k[..., out] = 0.0
    s = [np.einsum("thd,shd->hts", packed.rope_part(x, pos + n, rot, offset, inter, w),
                   packed.rope_part(k, pos + n, rot, offset, inter, w)) for n in (0, 7)]
    assert np.allclose(*s)


def test_rope_part_of_whole_heads_in_halves_is_plain_rope():
    rng = np.random.default_rng(2)
    x, pos = rng.standard_normal((7, 3, 32)), np.arange(7) * 5
    w = packed.part_frequencies(32, 1e4)
    y = packed.rope_part(x, pos, 32, 0, False, w)
    assert np.allclose(y, dense.rope_fwd(x, 1, 7, 1e4, pos))
    # interleaved: the same of columns dealt in turn
    deal = np.arange(32).reshape(2, 16).T.ravel()
    z = packed.rope_part(x[..., deal], pos, 32, 0, True, w)
    assert np.allclose(z, y[..., deal])


def test_interleaved_pairs_by_hand():
    w = packed.part_frequencies(4, 100.0)
    assert np.allclose(w, [1.0, 0.1])
    x = np.zeros((1, 1, 8))
    x[0, 0, 2], x[0, 0, 5] = 1.0, 1.0
    y = packed.rope_part(x, np.array([1]), 4, 2, True, w)[0, 0]
    assert np.allclose(y, [0, 0, np.cos(1), np.sin(1), -np.sin(0.1), np.cos(0.1), 0, 0])


def test_scaled_frequencies():
    w = packed.part_frequencies(32, 1e4)
    assert np.allclose(packed.part_frequencies(32, 1e4, "linear", 4.0), w / 4)
    b = packed.part_frequencies(32, 1e4, "base", 4.0)
    assert b[0] == 1.0 and np.isclose(b[-1], w[-1] / 4)
    # by parts: 4096 positions, a pair that makes more than 32 turns in them stays, one
    # of less than one is interpolated, and between a share of both
    p = packed.part_frequencies(64, 1e4, "parts", 8.0, 1.0, 32.0, 4096)
    w = packed.part_frequencies(64, 1e4)
    turns = 4096 * w / (2 * np.pi)
    assert np.allclose(p[turns >= 32], w[turns >= 32]) and np.any(turns >= 32)
    assert np.allclose(p[turns <= 1], w[turns <= 1] / 8) and np.any(turns <= 1)
    mid = np.flatnonzero((turns > 1) & (turns < 32))
    g = (turns[mid] - 1) / 31
    assert mid.size and np.allclose(p[mid] / w[mid], g + (1 - g) / 8)
    assert np.allclose(packed.part_frequencies(8, 1e4, pair_factors=[1, 2, 4, 8]),
                       packed.part_frequencies(8, 1e4) / [1, 2, 4, 8])


@pytest.mark.parametrize("rot,offset,inter", PARTS)
def test_rope_part_backward_finite_differences(rot, offset, inter):
    rng = np.random.default_rng(3)
    x, dy, pos = rng.standard_normal((4, 2, 16)), rng.standard_normal((4, 2, 16)), np.arange(4) * 3
    w = packed.part_frequencies(rot, 50.0)

    def f():
        return float((packed.rope_part(x, pos, rot, offset, inter, w, 1.3) * dy).sum())
    got = packed.rope_part(dy, pos, rot, offset, inter, w, 1.3, backward=True)
    # (the columns that pass through are not scaled)
    assert rel_err(got.ravel(), central_diff(f, x, np.arange(x.size))) <= 1e-6
