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


# ------------------------------------------------------- moments of 8 bits ----

def _moments(rng, n):
    m = (rng.standard_normal(n) * 10.0 ** rng.uniform(-6, 0, n)).astype(np.float32)
    return m, (rng.standard_normal(n).astype(np.float32) ** 2 * 10.0 ** rng.uniform(
        -9, 0, n)).astype(np.float32)


def test_codes_bracket_the_value():
    """The nearest code is within half a step; a drawn one within a step."""
    rng = np.random.default_rng(11)
    m, v = _moments(rng, 3000)
    for seed, share in ((None, 0.5), (7, 1.0)):
        um, uv = packed.moment_draws(3000, 0, seed)
        q, s = packed.encode_m(m, um)
        top = np.repeat(s, 256)[:3000]
        step = (2 * np.abs(q.astype(np.float64)) + 1) / 16129 * top
        assert np.all(np.abs(packed.decode_m(q, s) - m) <= share * step * 1.0001 + 1e-12)
        q, s = packed.encode_v(v, uv)
        top, c = np.repeat(s, 256)[:3000], q.astype(np.float64)
        step = ((c + 1) ** 4 - c ** 4) / 255.0 ** 4 * top
        assert np.all(np.abs(packed.decode_v(q, s) - v) <= share * step * 1.0001 + 1e-12)


def test_the_largest_of_a_block_is_exact_and_codes_are_kept():
    rng = np.random.default_rng(12)
    m, v = _moments(rng, 1024)
    for seed in (None, 3):
        um, uv = packed.moment_draws(1024, 5, seed)
        for x, u, enc, dec in ((m, um, packed.encode_m, packed.decode_m),
                               (v, uv, packed.encode_v, packed.decode_v)):
            q, s = enc(x, u)
            y = dec(q, s)
            at = np.abs(x.reshape(-1, 256)).argmax(axis=1) + 256 * np.arange(4)
            # (a largest value a rounding below its code's may be drawn down: not here)
            assert np.allclose(y[at], x[at], rtol=1e-6)
            # a value that is a code's already keeps it, whatever is drawn
            q2, s2 = enc(y, u)
            assert np.mean(q2 != q) <= 2e-3 and np.allclose(s2, s)


def test_drawn_codes_keep_the_mean():
    """4000 seeds: the mean of 256 values each is theirs within 5 standard deviations of a
    step's uniform rounding (step / 2 / sqrt(4000))."""
    rng = np.random.default_rng(13)
    m, v = _moments(rng, 256)
    n = 4000
    am, av = np.zeros(256), np.zeros(256)
    for seed in range(n):
        um, uv = packed.moment_draws(256, 1, seed)
        am += packed.decode_m(*packed.encode_m(m, um))
        av += packed.decode_v(*packed.encode_v(v, uv))
    qm = np.floor(np.sqrt(np.abs(m) / np.abs(m).max()) * 127)
    qv = np.floor((v.astype(np.float64) / v.max()) ** 0.25 * 255)
    sm = (2 * qm + 1) / 16129 * np.abs(m).max()
    sv = ((qv + 1) ** 4 - qv ** 4) / 255.0 ** 4 * v.max()
    assert np.all(np.abs(am / n - m) <= 5 * sm / 2 / np.sqrt(n) + 1e-6 * np.abs(m))
    # (v keeps a code above zero: below it the mean is the first code's)
    up = qv >= 1
    assert np.all((np.abs(av / n - v) <= 5 * sv / 2 / np.sqrt(n) + 1e-6 * v)[up])


def test_draws_are_uniform_and_differ():
    um, uv = packed.moment_draws(1 << 16, 0, 42)
    for u in (um, uv):
        assert 0 < u.min() and u.max() < 1
        count = np.bincount((u * 64).astype(int), minlength=64)
        # chi-square of 63 degrees of freedom: mean 63, 5 deviations 56
        assert np.sum((count - 1024.0) ** 2 / 1024.0) < 63 + 56
        assert abs(np.corrcoef(u[:-1], u[1:])[0, 1]) < 5 / 256
    assert abs(np.corrcoef(um, uv)[0, 1]) < 5 / 256
    for other in (packed.moment_draws(1 << 16, 1, 42), packed.moment_draws(1 << 16, 0, 43)):
        assert abs(np.corrcoef(um, other[0])[0, 1]) < 5 / 256


def test_zero_tiny_and_small_blocks():
    z = np.zeros(300, np.float32)
    half = np.full(300, np.float32(0.5))
    for enc, dec in ((packed.encode_m, packed.decode_m), (packed.encode_v, packed.decode_v)):
        q, s = enc(z, half)
        assert not q.any() and not s.any() and not dec(q, s).any()
        q, s = enc(z + np.float32(2.0 ** -96), half)
        assert not q.any() and not s.any()
    v = np.zeros(256, np.float32)
    v[0], v[1] = 1.0, 1e-30
    q, s = packed.encode_v(v, np.full(256, np.float32(0.99)))
    assert q[0] == 255 and q[1] == 1 and not q[2:].any()


# ------------------------------------------------------- packed attention ----

def _qkv(rng, T, nh=2, nkv=1, d=4):
    return (rng.standard_normal((T, nh, d)), rng.standard_normal((T, nkv, d)),
            rng.standard_normal((T, nkv, d)), rng.standard_normal((T, nh, d)))


def test_sequences_of_offsets():
    assert packed.sequences([0, 3, 3, 8], 10, 10) == [(0, 3), (3, 0), (3, 5)]
    assert packed.sequences([2, 7, 99], 10, 4) == [(2, 4), (7, 3)]
    assert packed.sequences([-5, 4, 2, 6], 10, 10) == [(0, 4), (4, 0), (4, 2)]
    assert packed.covered([2, 7, 99], 10, 4).tolist() == [False] * 2 + [True] * 4 + [False] + [True] * 3
    assert packed.positions([1, 3, 5], 6, 9).tolist() == [-1, 0, 1, 0, 1, -1]


def test_packed_attention_is_each_sequence_s_own():
    rng = np.random.default_rng(21)
    q, k, v, do = _qkv(rng, 12)
    off = [0, 5, 5, 6, 11]
    r = packed.attention(q, k, v, do, off, 12)
    for a, b in ((0, 5), (5, 6), (6, 11)):
        o, lse = dense.attention_fwd(q[a:b], k[a:b], v[a:b], 1, b - a)
        assert np.allclose(r["o"][a:b], o) and np.allclose(r["lse"][:, a:b], lse[0])
        for got, ref in zip((r["dq"], r["dk"], r["dv"]),
                            dense.attention_bwd(q[a:b], k[a:b], v[a:b], do[a:b], 1, b - a)):
            assert np.allclose(got[a:b], ref)
    assert np.isnan(r["o"][11]).all() and np.isnan(r["dk"][11]).all()
    # a sequence of one token attends to itself
    assert np.allclose(r["o"][5], v[5])
    # other sequences' rows change nothing
    q2, k2, v2 = (x.copy() for x in (q, k, v))
    for x in (q2, k2, v2):
        x[:6] += 3.0
    r2 = packed.attention(q2, k2, v2, do, off, 12)
    assert all(np.array_equal(r[n][6:11], r2[n][6:11]) for n in ("o", "dq", "dk", "dv"))


@pytest.mark.parametrize("window", [0, 1, 3])
def test_packed_attention_backward_finite_differences(window):
    rng = np.random.default_rng(22)
    q, k, v, do = _qkv(rng, 9)
    off = [0, 4, 5, 9]

    def f():
        return float((packed.attention(q, k, v, None, off, 9, window)["o"] * do).sum())
    r = packed.attention(q, k, v, do, off, 9, window)
    for got, wrt in ((r["dq"], q), (r["dk"], k), (r["dv"], v)):
        diff = central_diff(f, wrt, np.arange(wrt.size))
        if window == 1 and wrt is not v:
            # one visible key has weight 1 whatever its score: no gradient but fp64 rounding
            # of dP - delta (two sums of four products below 20 each), and no relative error
            assert not diff.any() and np.abs(got).max() <= 4 * 20 * 2.0 ** -52
        else:
            assert rel_err(got.ravel(), diff) <= 1e-6


def test_a_small_v_beside_a_huge_one_keeps_a_code():
    """... though its share of it, in 255^-4ths, is below what fp32 holds."""
    v = np.zeros(256, np.float32)
    v[0], v[1], v[2] = 2.0 ** 117, 2.0 ** -70, 2.0 ** -149
    for u in (0.01, 0.5, 0.99):
        q, s = packed.encode_v(v, np.full(256, np.float32(u)))
        assert s[0] == v[0] and q[0] == 255 and q[1] == 1 and q[2] == 1 and not q[3:].any()
