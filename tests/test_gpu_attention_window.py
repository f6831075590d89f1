"""GPU parity of forge_attention_window_fwd / _bwd with the fp64 oracle.

Three kinds of checks:
  * which pairs see each other, exactly: with zero scores every visible key has
    the same weight, so a row's log-sum-exp is the log of their number, and an
    upstream gradient on one row leaves dk and dv on its visible keys alone;
  * every element of o, dq, dk, dv within what the roundings to bf16 may move
    it (oracle.branch works that out; fp32 sums add 1e-5 of the same terms);
  * the whole of each output, whose roundings are independent, to 2^-7.
"""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import branch
from gpu_util import rel_fro, dev_bf16, host_f64, banner

pytestmark = pytest.mark.gpu

CASES = [
    # batch, seq, heads, kv heads, head_dim, window, sinks, lens
    (1, 1, 4, 1, 128, 1, 0, None),
    (1, 1, 2, 2, 64, 5, 3, None),
    (2, 130, 4, 2, 64, 1, 0, None),
    (2, 130, 4, 2, 128, 1, 4, None),
    (1, 257, 4, 2, 64, 64, 2, None),
    (1, 257, 4, 1, 128, 65, 0, None),
    (3, 333, 6, 2, 64, 128, 4, (333, 200, 45)),
    (3, 200, 4, 2, 128, 31, 70, (0, 1, 199)),
    (1, 700, 4, 1, 64, 33, 130, None),
    (1, 700, 4, 1, 128, 33, 100, None),
    (2, 320, 8, 2, 128, 320, 0, (64, 320)),
    (1, 900, 3, 1, 128, 300, 64, None),
    (1, 1100, 8, 8, 64, 200, 65, (1000,)),
    (4, 96, 2, 1, 64, 7, 1, (96, 95, 33, 0)),
    (1, 2050, 2, 1, 128, 513, 16, None),
    (1, 2050, 2, 1, 64, 100, 3, (1987,)),
    # many heads to a kv head: the key tiles' queries are walked round their window
    (1, 700, 8, 1, 128, 100, 3, None),
    (2, 450, 16, 1, 64, 90, 70, (450, 391)),
    (1, 1300, 16, 2, 128, 400, 0, None),
    # as many blocks of 256 queries as CUs, and more
    (2, 530, 48, 4, 64, 150, 66, (530, 301)),
    (1, 420, 128, 16, 128, 90, 2, None),
    # more blocks of 64 queries than run at once: the forward's blocks of 128, and the
    # last one's many rounds of 64
    (3, 200, 90, 6, 64, 37, 3, (200, 129, 0)),
    (1, 700, 96, 4, 64, 33, 130, (513,)),
    (17, 64, 64, 8, 64, 64, 0, None),
    (9, 450, 60, 6, 64, 120, 2, (450, 449, 0, 64, 65, 63, 300, 128, 129)),
    # up to four of them on a CU (head dim 64)
    (3, 200, 48, 12, 64, 37, 3, (200, 129, 0)),
    (2, 333, 24, 6, 128, 100, 70, (333, 65)),
    (1, 129, 180, 12, 64, 5, 0, None),
    (5, 65, 30, 2, 128, 3, 1, (65, 64, 1, 33, 65)),
    (2, 700, 24, 4, 64, 33, 130, (700, 513)),
    # as many blocks of 128 queries as run at once, with many key tiles
    (3, 600, 10, 2, 128, 450, 70, (600, 333, 0)),
    (1, 1100, 20, 4, 128, 1100, 0, None),
    # many key tiles and many sums beside few blocks of 64 queries
    (1, 1500, 8, 2, 64, 1000, 0, (1437,)),
    (1, 1100, 6, 3, 128, 1100, 0, None),
    # one tile of keys
    (2, 64, 4, 2, 64, 20, 3, (64, 0)),
    (3, 50, 6, 2, 128, 50, 0, (50, 33, 1)),
    # a score gradient beyond the memory-side cache: stored past it
    (1, 3500, 20, 4, 64, 2000, 2, None),
    (1, 3500, 20, 2, 128, 1990, 0, (3333,)),
]


def _dev(lens):
    import torch
    return None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")


def _call(B, S, nh, nkv, d, W, sinks, lens, qkv, do=None):
    """(o, lse, dqkv) on the GPU, every output and the scratch filled with NaN before."""
    import torch
    from paper_2609_13645_amd import _lib
    cfg = _lib.AttnWindowCfg(B, S, nh, nkv, d, W, sinks)
    nan = float("nan")
    o = torch.full((B * S, nh * d), nan, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, nh, S), nan, device="cuda")
    _lib.forge_attention_window_fwd(cfg, qkv, _dev(lens), o, lse)
    dqkv = None
    if do is not None:
        dqkv = torch.full_like(qkv, nan)
        n = _lib.forge_attention_window_bwd_workspace_bytes(cfg)
        ws = torch.full((n // 4,), nan, device="cuda")
        _lib.forge_attention_window_bwd(cfg, qkv, _dev(lens), o, lse, do, dqkv, ws)
    torch.cuda.synchronize()
    return o, lse, dqkv


def _split(x, nh, nkv, d):
    hq, hkv = nh * d, nkv * d
    T = x.shape[0]
    return (x[:, :hq].reshape(T, nh, d), x[:, hq:hq + hkv].reshape(T, nkv, d),
            x[:, hq + hkv:].reshape(T, nkv, d))


def _pad_rows(B, S, lens):
    n = [S] * B if lens is None else lens
    return np.concatenate([np.arange(S) >= k for k in n])


@pytest.mark.parametrize("B,S,nh,nkv,d,W,sinks,lens", CASES)
def test_parity(B, S, nh, nkv, d, W, sinks, lens):
    banner(f"window attention B={B} S={S} nh={nh} nkv={nkv} d={d} W={W} sinks={sinks} lens={lens}")
    rng = np.random.default_rng(S * 7 + d + W)
    T, hq, hkv = B * S, nh * d, nkv * d
    qkv_b = fi.to_bf16_bits(rng.standard_normal((T, hq + 2 * hkv), dtype=np.float32))
    do_b = fi.to_bf16_bits(rng.standard_normal((T, hq), dtype=np.float32))
    x, g = fi.bf16_bits_to_f64(qkv_b), fi.bf16_bits_to_f64(do_b)
    pad = _pad_rows(B, S, lens)
    # what stands behind a row's tokens is not read: NaN there
    qkv_b[pad] = do_b[pad] = 0x7FC0
    o, lse, dqkv = _call(B, S, nh, nkv, d, W, sinks, lens, dev_bf16(qkv_b), dev_bf16(do_b))
    q, k, v = _split(x, nh, nkv, d)
    r = branch.window_attention(q, k, v, g.reshape(T, nh, d), B, S, W, sinks, lens)
    got = dict(zip(("dq", "dk", "dv"), _split(host_f64(dqkv), nh, nkv, d)),
               o=host_f64(o).reshape(T, nh, d))
    lse = host_f64(lse)
    assert np.array_equal(np.isneginf(lse), np.isneginf(r["lse"]))
    seen = np.isfinite(r["lse"])
    assert np.allclose(lse[seen], r["lse"][seen], rtol=0, atol=1e-5)
    for n, y in got.items():
        assert np.all(y[pad] == 0.0), n
        # (one visible key has no score gradient: what is left is dP - delta)
        slack = 1e-5 * np.max(np.abs(g)) * np.max(np.abs(x)) ** 2
        off, bound = np.abs(y - r[n]), 1.02 * r["err_" + n] + slack
        assert np.all(off <= bound), f"{n}: {float(np.max(off / bound)):.2f} of its bound"
        if np.linalg.norm(r[n]) > 1e-6 * np.linalg.norm(r["o"]):
            assert rel_fro(y, r[n]) <= 2.0 ** -7, n


@pytest.mark.parametrize("B,S,nh,nkv,d,W,sinks,lens", CASES + [
    (1, 4096, 2, 1, 64, 1000, 200, None), (1, 5000, 1, 1, 128, 129, 1, None),
    (2, 3000, 2, 2, 128, 64, 64, (3000, 2940))])
def test_visible_pairs_exactly(B, S, nh, nkv, d, W, sinks, lens):
    """Zero scores: lse is the log of the number of visible keys; d_o on one row per
    head: dv is nonzero on that row's visible keys and nowhere else, dk with it."""
    import torch
    banner(f"visible pairs B={B} S={S} d={d} W={W} sinks={sinks} lens={lens}")
    T, hq, hkv = B * S, nh * d, nkv * d
    rng = np.random.default_rng(S + W)
    n_of = [S] * B if lens is None else list(lens)
    qkv = torch.zeros((T, hq + 2 * hkv), dtype=torch.bfloat16, device="cuda")
    qkv[:, hq + hkv:] = torch.randn((T, hkv), device="cuda").to(torch.bfloat16)
    vis = [branch.visible(n, W, sinks) for n in n_of]
    _, lse, _ = _call(B, S, nh, nkv, d, W, sinks, lens, qkv)
    count = np.exp(host_f64(lse))
    for b, n in enumerate(n_of):
        assert np.all(np.isneginf(host_f64(lse)[b, :, n:]))
        if n:
            want = vis[b].sum(axis=1)
            # fp32 log: 2^-22 of a value below 10
            assert np.all(np.abs(count[b, :, :n] - want) <= 1e-5 * want)
    # edges of tiles and of the window, and some rows between
    probes = sorted({0, W - 1, W, W + 31, W + 63, S - 1, S // 2, 63, 64, sinks,
                     *rng.integers(0, S, 6).tolist()})
    probes = [i for i in probes if 0 <= i < S]
    grp = nh // nkv
    for at in range(0, len(probes), nkv):
        rows = probes[at:at + nkv]                 # one probed row for each kv head
        do = torch.zeros((T, hq), dtype=torch.bfloat16, device="cuda")
        for m, i in enumerate(rows):
            for b in range(B):
                do[b * S + i, m * grp * d:(m * grp + 1) * d] = 1.0
        q1 = qkv.clone()
        q1[:, :hq] = 2.0 ** -10                    # scores stay equal (k is zero), dk is not
        _, _, dqkv = _call(B, S, nh, nkv, d, W, sinks, lens, q1, do)
        _, dk, dv = _split(host_f64(dqkv), nh, nkv, d)
        for m, i in enumerate(rows):
            for b, n in enumerate(n_of):
                want = np.zeros(S, bool)
                if i < n:
                    want[:n] = vis[b][i]
                assert np.array_equal((dv[b * S:(b + 1) * S, m] != 0).all(axis=1), want), (b, i)
                assert np.array_equal((dv[b * S:(b + 1) * S, m] != 0).any(axis=1), want), (b, i)
                some = (dk[b * S:(b + 1) * S, m] != 0).any(axis=1)
                assert not np.any(some & ~want), (b, i)
                if want.sum() > 1:
                    # (a key whose dP happens to equal delta has none)
                    assert some.sum() >= want.sum() - 1 - want.sum() // 50, (b, i)


@pytest.mark.parametrize("S,nh,nkv,d", [(129, 4, 2, 64), (700, 4, 1, 128)])
def test_window_of_the_whole_row_is_causal_attention(S, nh, nkv, d):
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"window >= seq S={S} d={d}")
    rng = np.random.default_rng(S)
    qkv = dev_bf16(fi.to_bf16_bits(rng.standard_normal((S, (nh + 2 * nkv) * d), dtype=np.float32)))
    cfg = _lib.AttnCfg(1, S, nh, nkv, d)
    o = torch.empty((S, nh * d), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((1, nh, S), device="cuda")
    _lib.forge_attention_fwd(cfg, qkv, o, lse)
    for W, sinks in ((S, 0), (1 << 30, 1 << 30), (1, S)):
        o2, lse2, _ = _call(1, S, nh, nkv, d, W, sinks, None, qkv)
        assert rel_fro(host_f64(o2), host_f64(o)) <= 2.0 ** -8
        assert float((lse2 - lse).abs().max()) <= 1e-5


def test_the_end_of_a_row_of_over_4_gb():
    """The last rows depend on the last ones alone: those of the oracle over these."""
    import torch
    S, nh, nkv, d, W, n = (1 << 22) + 100, 2, 1, 128, 70, 600
    banner(f"window attention S={S} nh={nh} nkv={nkv} d={d} W={W}")
    qkv = torch.randn((S, (nh + 2 * nkv) * d), dtype=torch.bfloat16, device="cuda")
    do = torch.randn((S, nh * d), dtype=torch.bfloat16, device="cuda")
    o, lse, dqkv = (t[..., -n:, :] if t.dim() == 2 else t[..., -n:]
                    for t in _call(1, S, nh, nkv, d, W, 0, None, qkv, do))
    x, g = host_f64(qkv[-n:]), host_f64(do[-n:])
    q, k, v = _split(x, nh, nkv, d)
    r = branch.window_attention(q, k, v, g.reshape(n, nh, d), 1, n, W, 0, None)
    got = dict(zip(("dq", "dk", "dv"), _split(host_f64(dqkv), nh, nkv, d)),
               o=host_f64(o).reshape(n, nh, d))
    assert np.allclose(host_f64(lse)[..., W:], r["lse"][..., W:], rtol=0, atol=1e-5)
    for name, y in got.items():
        slack = 1e-5 * np.max(np.abs(g)) * np.max(np.abs(x)) ** 2
        off, bound = np.abs(y - r[name])[W:], (1.02 * r["err_" + name] + slack)[W:]
        assert np.all(off <= bound), f"{name}: {float(np.max(off / bound)):.2f} of its bound"


def test_lens_outside_the_row_are_clamped():
    import torch
    banner("window attention clamped lens")
    B, S, nh, nkv, d = 3, 100, 2, 1, 64
    qkv = torch.randn((B * S, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((B * S, nh * d), device="cuda").to(torch.bfloat16)
    a = _call(B, S, nh, nkv, d, 20, 2, (-7, 2 ** 31 - 1, 50), qkv, do)
    b = _call(B, S, nh, nkv, d, 20, 2, (0, S, 50), qkv, do)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_large_scores_and_hidden_infinities():
    """Scores of thousands, of both signs, keep their softmax; a hidden key's
    infinity or NaN changes no row that does not see it (its value's may)."""
    import torch
    banner("window attention large scores")
    S, d, W = 300, 64, 70
    rng = np.random.default_rng(5)
    x = rng.standard_normal((S, 3 * d))
    x[:, :2 * d] *= 30.0
    qkv_b = fi.to_bf16_bits(x.astype(np.float32))
    x64 = fi.bf16_bits_to_f64(qkv_b)
    q, k, v = _split(x64, 1, 1, d)
    r = branch.window_attention(q, k, v, None, 1, S, W, 3)
    o, lse, _ = _call(1, S, 1, 1, d, W, 3, None, dev_bf16(qkv_b))
    assert np.allclose(host_f64(lse), r["lse"], rtol=2e-6, atol=0)
    # scores of up to 30^2 * 8 * 3 = 2^14 carry 2^-24 of themselves, into the exponent
    off = np.abs(host_f64(o).reshape(S, 1, d) - r["o"])
    assert np.all(off <= 1.02 * r["err_o"] + 4 * 2.0 ** -10 * np.max(np.abs(x64[:, 2 * d:])))
    bad = dev_bf16(qkv_b)
    bad[20, d:2 * d] = float("inf")
    bad[21, d:2 * d] = float("nan")
    o2, _, _ = _call(1, S, 1, 1, d, W, 3, None, bad)
    free = np.r_[np.arange(20), np.arange(21 + W, S)]
    assert torch.equal(o2[free], o[free])


def test_results_repeat_bit_for_bit():
    import torch
    banner("window attention determinism")
    B, S, nh, nkv, d = 2, 900, 8, 2, 128
    qkv = torch.randn((B * S, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((B * S, nh * d), device="cuda").to(torch.bfloat16)
    first = _call(B, S, nh, nkv, d, 100, 70, (900, 640), qkv, do)
    for _ in range(2):
        again = _call(B, S, nh, nkv, d, 100, 70, (900, 640), qkv, do)
        assert all(torch.equal(a, b) for a, b in zip(again, first))


@pytest.mark.parametrize("B,S,nh,nkv,d,W,sinks,lens", [
    (3, 200, 4, 2, 64, 40, 3, (200, 90, 0)),
    (3, 200, 4, 2, 128, 40, 3, (200, 90, 0)),
    # sums of partials: of splits, of the chunks of what the sinks see
    (2, 1000, 8, 2, 64, 300, 70, (333, 1000)),
    (2, 1500, 8, 2, 128, 100, 70, (1409, 1500)),
    (2, 700, 48, 4, 128, 64, 0, (65, 700)),
])
def test_infinities_stay_in_their_batch_row_and_kv_head(B, S, nh, nkv, d, W, sinks, lens):
    """A token's NaN or infinity, in q, k, v or d_o of the first heads of batch row b, leaves
    the other batch rows and kv heads as they are, bit for bit, and padding rows zeros."""
    import torch
    banner(f"window attention infinities B={B} S={S} nh={nh} nkv={nkv} d={d} W={W} sinks={sinks}")
    hq, hkv, grp = nh * d, nkv * d, nh // nkv
    b = 1 if lens[1] < S else 0
    qkv = torch.randn((B * S, hq + 2 * hkv), device="cuda").to(torch.bfloat16)
    do = torch.randn((B * S, hq), device="cuda").to(torch.bfloat16)
    clean = _call(B, S, nh, nkv, d, W, sinks, lens, qkv, do)
    pad = torch.from_numpy(_pad_rows(B, S, lens)).cuda()
    # rows that share a tile of keys with the padding, and the row's first
    at = [b * S, b * S + lens[b] - 1]
    for what, col in (("q", 0), ("k", hq), ("v", hq + hkv), ("d_o", None)):
        for value in (float("inf"), float("nan")):
            x, g = qkv.clone(), do.clone()
            if col is None:
                g[at, :d] = value
            else:
                x[at, col:col + d] = value
            o, lse, dqkv = _call(B, S, nh, nkv, d, W, sinks, lens, x, g)
            assert not o[pad].any() and not dqkv[pad].any(), (what, value)
            other = torch.arange(B * S, device="cuda") // S != b
            assert torch.equal(o[other], clean[0][other]), (what, value)
            assert torch.equal(dqkv[other], clean[2][other]), (what, value)
            assert torch.equal(o[:, grp * d:], clean[0][:, grp * d:]), (what, value)
            assert torch.equal(lse[:, grp:], clean[1][:, grp:]), (what, value)
            for lo, hi in ((grp * d, hq), (hq + d, hq + hkv), (hq + hkv + d, hq + 2 * hkv)):
                assert torch.equal(dqkv[:, lo:hi], clean[2][:, lo:hi]), (what, value)
            # (the row itself does show it)
            assert not torch.isfinite(dqkv[b * S:b * S + lens[b]]).all(), (what, value)


@pytest.mark.parametrize("d", [64, 128])
def test_backward_of_a_forward_result_that_is_not_finite(d):
    """The same of o and lse as the backward takes them, in both forms of the row sums."""
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"window attention infinities of o and lse d={d}")
    for B, S, nh, nkv, W, lens in ((2, 200, 4, 2, 40, (200, 90)), (2, 1000, 48, 4, 300, (650, 999))):
        hq, hkv, grp = nh * d, nkv * d, nh // nkv
        qkv = torch.randn((B * S, hq + 2 * hkv), device="cuda").to(torch.bfloat16)
        do = torch.randn((B * S, hq), device="cuda").to(torch.bfloat16)
        o, lse, clean = _call(B, S, nh, nkv, d, W, 3, lens, qkv, do)
        cfg = _lib.AttnWindowCfg(B, S, nh, nkv, d, W, 3)
        pad = torch.from_numpy(_pad_rows(B, S, lens)).cuda()
        at = S + lens[1] - 1
        for bad in (float("inf"), float("nan"), float("-inf")):
            o2, lse2 = o.clone(), lse.clone()
            o2[at - 5, :d] = bad
            lse2[1, 0, lens[1] - 1] = bad
            got = torch.full_like(qkv, float("nan"))
            ws = torch.full((_lib.forge_attention_window_bwd_workspace_bytes(cfg) // 4,),
                            float("nan"), device="cuda")
            _lib.forge_attention_window_bwd(cfg, qkv, _dev(lens), o2, lse2, do, got, ws)
            torch.cuda.synchronize()
            assert not got[pad].any()
            assert torch.equal(got[:S], clean[:S])
            for lo, hi in ((grp * d, hq), (hq + d, hq + hkv), (hq + hkv + d, hq + 2 * hkv)):
                assert torch.equal(got[:, lo:hi], clean[:, lo:hi])


@pytest.mark.parametrize("B,S,nh,nkv,d,W,sinks,lens", [
    # windows and sinks that reach the end of the sequence: before, at and behind the key
    # tile from which it cuts them, with an odd number of 32 queries and an even one
    (1, 700, 4, 1, 64, 400, 130, None),
    (1, 161, 4, 2, 128, 90, 70, (150,)),
    (2, 97, 2, 1, 64, 60, 1, None),
    (1, 1100, 6, 3, 64, 700, 1100, (1037,)),
    (1, 640, 4, 1, 128, 320, 64, None),
    (2, 640, 4, 4, 64, 2, 321, (640, 577)),
    (1, 450, 8, 2, 128, 449, 385, None),
    # more of the score gradient than the memory-side cache holds
    (1, 2050, 64, 4, 64, 1500, 2, None),
    (1, 2050, 64, 4, 128, 2050, 0, (2011,)),
])
def test_parity_where_the_end_of_the_sequence_cuts_windows(B, S, nh, nkv, d, W, sinks, lens):
    test_parity(B, S, nh, nkv, d, W, sinks, lens)
