"""GPU parity of forge_attention_packed_plan / _fwd / _bwd with the fp64 oracle.

Three kinds of checks:
  * which pairs see each other, exactly: with zero scores every visible key has
    the same weight, so a row's log-sum-exp is the log of their number, and an
    upstream gradient on one row leaves dv on its visible keys alone;
  * every element of o, dq, dk, dv within what the roundings to bf16 may move
    it (oracle.branch works that out; fp32 sums add 1e-5 of the same terms);
  * the whole of each output, whose roundings are independent, to 2^-7.
Rows of no sequence hold NaN in every input, and keep what every output held.
"""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import packed
from gpu_util import rel_fro, dev_bf16, host_f64, banner

pytestmark = pytest.mark.gpu

CASES = [
    # lens, rows before the first, rows behind the last, heads, kv heads, head_dim, window
    ([1], 0, 0, 4, 1, 128, 0),
    ([1], 0, 3, 2, 2, 64, 1),
    ([0], 0, 5, 2, 1, 64, 0),
    ([1, 1, 0, 2, 1, 3], 2, 1, 4, 2, 128, 0),
    ([333, 1, 0, 200, 77], 0, 0, 6, 2, 64, 0),
    ([65, 129, 63], 0, 0, 4, 2, 64, 0),
    ([64, 128, 256, 64], 0, 0, 4, 4, 128, 0),
    ([63, 127, 255, 65, 31, 33], 7, 9, 3, 1, 128, 0),
    ([700, 3, 1100], 0, 40, 8, 2, 128, 0),
    ([1100, 90, 513], 0, 0, 16, 2, 64, 0),
    ([130, 257, 64, 5], 1, 0, 4, 2, 128, 64),
    ([513, 900, 30, 64], 0, 65, 8, 1, 64, 100),
    ([700, 700], 0, 0, 4, 4, 128, 1),
    ([2050, 17, 333], 0, 0, 4, 1, 128, 513),
    ([2050, 700], 0, 3, 2, 1, 64, 65),
    ([16] * 100 + [0, 0, 7], 0, 0, 8, 2, 64, 0),
    ([5, 40, 1, 90, 0, 33, 70] * 15, 3, 3, 32, 8, 128, 0),
    ([1500, 60, 900], 0, 0, 20, 4, 64, 0),
    ([400] * 9, 0, 0, 48, 6, 128, 300),
    ([3500, 500], 0, 0, 20, 4, 64, 0),
    # (many blocks of key tiles: of two waves, then of one)
    ([5, 40, 1, 90, 0, 33, 70] * 15, 3, 3, 32, 8, 64, 0),
    ([130, 200, 64, 5, 90] * 8, 0, 2, 48, 24, 64, 40),
    ([5, 40, 1, 90, 0, 33, 70] * 15, 0, 5, 64, 16, 64, 0),
    ([130, 200, 64, 5, 90] * 8, 1, 0, 64, 32, 64, 40),
    ([5, 40, 1, 90, 0, 33, 70] * 15, 0, 5, 64, 16, 128, 0),
    ([130, 200, 64, 5, 90] * 8, 1, 0, 64, 32, 128, 40),
    # (many of four waves)
    ([2500, 60, 900, 40], 2, 3, 16, 8, 64, 0),
    ([1300, 60, 900, 40], 0, 0, 16, 16, 128, 0),
    # (one long sequence: blocks of 128 whose key tiles are in two groups, for every group of heads)
    ([1500, 700, 300], 0, 1, 16, 4, 128, 0),
    ([3500, 700], 0, 0, 8, 4, 128, 0),
    ([3500, 700], 2, 0, 9, 3, 128, 0),
    # (and dQ blocks of 256)
    ([1500, 1300], 0, 0, 32, 8, 128, 0),
    ([2500, 900, 700], 0, 0, 16, 8, 128, 0),
    ([1300, 1100], 0, 5, 36, 12, 128, 0),
    ([1500, 1300], 3, 0, 32, 8, 64, 0),
    ([2500, 900, 700], 0, 0, 16, 8, 64, 0),
    # (the same of sequences alike; a long one among many; and within a window)
    ([1300] * 3, 0, 0, 32, 8, 128, 0),
    ([1290, 1300, 1300], 1, 0, 16, 8, 128, 0),
    ([1300] * 3, 0, 2, 36, 12, 128, 0),
    ([1300] * 3, 0, 0, 32, 8, 64, 0),
    ([1300] * 3, 0, 0, 16, 8, 64, 0),
    ([400] * 9, 0, 0, 24, 8, 128, 0),
    ([40, 3, 61] * 12 + [2100] + [17, 29] * 5, 0, 0, 6, 2, 128, 0),
    ([40, 3, 61] * 12 + [2100] + [17, 29] * 5, 0, 0, 16, 8, 128, 25),
]


def offsets_of(lens, before):
    return (before + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)


class Call:
    """Buffers of one packed call; outputs and scratch filled with NaN, or a given value."""

    def __init__(self, off, tokens, max_seq, nh, nkv, d, window, qkv, do=None, fill=float("nan")):
        import torch
        from paper_2609_13645_amd import _lib
        self.L = _lib
        self.cfg = _lib.attn_packed_cfg(dict(tokens=tokens, n_seqs=len(off) - 1, max_seq=max_seq,
                                             n_heads=nh, n_kv_heads=nkv, head_dim=d, window=window))
        self.off = torch.from_numpy(np.asarray(off, np.int32)).cuda()
        f = lambda *s, dt=torch.bfloat16: torch.full(s, fill, dtype=dt, device="cuda")
        self.qkv, self.do = qkv, do
        self.plan = torch.full((_lib.forge_attention_packed_plan_bytes(self.cfg),), 0x7F,
                               dtype=torch.uint8, device="cuda")
        self.pos = torch.full((tokens,), -7, dtype=torch.int32, device="cuda")
        self.o, self.lse = f(tokens, nh * d), f(nh, tokens, dt=torch.float32)
        self.dqkv = None
        if do is not None:
            self.dqkv = f(tokens, (nh + 2 * nkv) * d)
            n = _lib.forge_attention_packed_bwd_workspace_bytes(self.cfg)
            self.ws = torch.full((n // 4,), float("nan"), device="cuda")

    def run(self, stream=None, plan=True):
        L, c, s = self.L, self.cfg, stream
        if plan:
            L.forge_attention_packed_plan(c, self.off, self.plan, self.pos, s)
        L.forge_attention_packed_fwd(c, self.plan, self.qkv, self.o, self.lse, s)
        if self.do is not None:
            L.forge_attention_packed_bwd(c, self.plan, self.qkv, self.o, self.lse, self.do,
                                         self.dqkv, self.ws, s)
        return self

    def results(self):
        return [t for t in (self.o, self.lse, self.dqkv) if t is not None]


def _split(x, nh, nkv, d):
    hq, hkv = nh * d, nkv * d
    T = x.shape[0]
    return (x[:, :hq].reshape(T, nh, d), x[:, hq:hq + hkv].reshape(T, nkv, d),
            x[:, hq + hkv:].reshape(T, nkv, d))


def _parity(off, T, max_seq, nh, nkv, d, W, seed):
    import torch
    rng = np.random.default_rng(seed)
    hq, hkv = nh * d, nkv * d
    qkv_b = fi.to_bf16_bits(rng.standard_normal((T, hq + 2 * hkv), dtype=np.float32))
    do_b = fi.to_bf16_bits(rng.standard_normal((T, hq), dtype=np.float32))
    x, g = fi.bf16_bits_to_f64(qkv_b), fi.bf16_bits_to_f64(do_b)
    inside = packed.covered(off, T, max_seq)
    qkv_b[~inside] = do_b[~inside] = 0x7FC0
    c = Call(off, T, max_seq, nh, nkv, d, W, dev_bf16(qkv_b), dev_bf16(do_b), fill=3.0).run()
    torch.cuda.synchronize()
    q, k, v = _split(x, nh, nkv, d)
    r = packed.attention(q, k, v, g.reshape(T, nh, d), off, max_seq, W)
    pos = packed.positions(off, T, max_seq)
    assert np.array_equal(c.pos.cpu().numpy()[inside], pos[inside])
    assert np.all(c.pos.cpu().numpy()[~inside] == -7)
    got = dict(zip(("dq", "dk", "dv"), _split(host_f64(c.dqkv), nh, nkv, d)),
               o=host_f64(c.o).reshape(T, nh, d))
    lse = host_f64(c.lse)
    assert np.all(lse[:, ~inside] == 3.0)
    assert np.allclose(lse[:, inside], r["lse"][:, inside], rtol=0, atol=1e-5)
    for n, y in got.items():
        assert np.all(y[~inside] == 3.0), n
        if not inside.any():
            continue
        # (one visible key has no score gradient: what is left is dP - delta)
        slack = 1e-5 * np.max(np.abs(g)) * np.max(np.abs(x)) ** 2
        off_by, bound = np.abs(y - r[n])[inside], 1.02 * r["err_" + n][inside] + slack
        assert np.all(off_by <= bound), f"{n}: {float(np.max(off_by / bound)):.2f} of its bound"
        if np.linalg.norm(r[n][inside]) > 1e-6 * np.linalg.norm(r["o"][inside]):
            assert rel_fro(y[inside], r[n][inside]) <= 2.0 ** -7, n


@pytest.mark.parametrize("lens,before,behind,nh,nkv,d,W", CASES)
def test_parity(lens, before, behind, nh, nkv, d, W):
    banner(f"packed attention {len(lens)} of {lens[:7]} +{before}+{behind} {nh}/{nkv}x{d} W={W}")
    off = offsets_of(lens, before)
    T = int(off[-1]) + behind
    _parity(off, T, max(1, max(lens)), nh, nkv, d, W, T + d)


@pytest.mark.parametrize("off,T,max_seq", [
    ([-5, 100, 90, 300, 2 ** 31 - 1], 400, 400),      # running maximum, cut to [0, tokens]
    ([0, 200, 260, 500], 500, 130),                   # longer than max_seq: its first rows
    ([50, -2 ** 31, 7], 60, 60),                      # nothing
    ([0, 500], 500, 1)])
def test_offsets_out_of_order_or_bounds(off, T, max_seq):
    """What they stand for is worked out before anything is read or written."""
    banner(f"packed attention offsets {off} max_seq={max_seq}")
    _parity(np.array(off, np.int64), T, max_seq, 4, 2, 64, 0, 5)


@pytest.mark.parametrize("lens,before,behind,nh,nkv,d,W", CASES + [
    ([5000], 0, 0, 1, 1, 128, 0), ([3000, 2940], 0, 60, 2, 2, 128, 64)])
def test_visible_pairs_exactly(lens, before, behind, nh, nkv, d, W):
    """Zero scores: lse is the log of the number of visible keys; d_o on some rows, one for
    each kv head: dv is nonzero on that row's visible keys and nowhere else."""
    import torch
    banner(f"packed visible pairs {lens[:7]} d={d} W={W}")
    off = offsets_of(lens, before)
    T, hq, hkv = int(off[-1]) + behind, nh * d, nkv * d
    rng = np.random.default_rng(T + W)
    qkv = torch.zeros((T, hq + 2 * hkv), dtype=torch.bfloat16, device="cuda")
    qkv[:, hq + hkv:] = torch.randn((T, hkv), device="cuda").to(torch.bfloat16)
    pos = packed.positions(off, T, T)
    inside = pos >= 0
    count = np.minimum(pos + 1, W or T)
    c = Call(off, T, max(1, max(lens)), nh, nkv, d, W, qkv).run()
    torch.cuda.synchronize()
    got = np.exp(host_f64(c.lse))
    # fp32 log: 2^-22 of a value below 10
    assert np.all(np.abs(got - count)[:, inside] <= 1e-5 * count[inside])
    if not inside.any():
        return
    # edges of sequences, of tiles and of the window, and some rows between
    edges = [int(o) + e for o in off for e in (-65, -64, -33, -1, 0, 31, 63, 64, W, W + 31)]
    probes = sorted({i for i in edges + rng.integers(0, T, 6).tolist() if 0 <= i < T and inside[i]})
    if len(probes) > 24:
        probes = sorted(rng.choice(probes, 24, replace=False).tolist())
    grp = nh // nkv
    for at in range(0, len(probes), nkv):
        rows = probes[at:at + nkv]
        do = torch.zeros((T, hq), dtype=torch.bfloat16, device="cuda")
        for m, i in enumerate(rows):
            do[i, m * grp * d:(m * grp + 1) * d] = 1.0
        c = Call(off, T, max(1, max(lens)), nh, nkv, d, W, qkv, do, fill=0.0).run()
        torch.cuda.synchronize()
        _, _, dv = _split(host_f64(c.dqkv), nh, nkv, d)
        for m, i in enumerate(rows):
            want = np.zeros(T, bool)
            want[i - count[i] + 1:i + 1] = True
            assert np.array_equal((dv[:, m] != 0).all(axis=1), want), i
            assert np.array_equal((dv[:, m] != 0).any(axis=1), want), i


@pytest.mark.parametrize("nh,nkv,d,W", [(4, 2, 64, 0), (4, 1, 128, 0), (8, 4, 64, 70)])
def test_one_sequence_is_a_batch_row(nh, nkv, d, W):
    """The outputs of forge_attention_window_fwd / _bwd of that row, but for what the two may
    round differently (running maxima and sums in another order): either is within the
    oracle's bound of the exact value, so they are within twice that of each other."""
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"packed one sequence d={d} W={W}")
    S = 700
    qkv = torch.randn((S, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((S, nh * d), device="cuda").to(torch.bfloat16)
    c = Call([0, S], S, S, nh, nkv, d, W, qkv, do).run()
    cfg = _lib.AttnWindowCfg(1, S, nh, nkv, d, W or S, 0)
    o, lse, dqkv = (torch.empty_like(t) for t in (c.o, c.lse, c.dqkv))
    ws = torch.empty(_lib.forge_attention_window_bwd_workspace_bytes(cfg), dtype=torch.uint8,
                     device="cuda")
    _lib.forge_attention_window_fwd(cfg, qkv, None, o, lse)
    _lib.forge_attention_window_bwd(cfg, qkv, None, o, lse, do, dqkv, ws)
    torch.cuda.synchronize()
    assert float((c.lse - lse).abs().max()) <= 2e-5
    q, k, v = _split(host_f64(qkv), nh, nkv, d)
    g = host_f64(do)
    r = packed.attention(q, k, v, g.reshape(S, nh, d), [0, S], S, W)
    slack = 1e-5 * np.max(np.abs(g)) * max(np.max(np.abs(x)) for x in (q, k, v)) ** 2
    both = [dict(zip(("dq", "dk", "dv"), _split(host_f64(t), nh, nkv, d)),
                 o=host_f64(u).reshape(S, nh, d)) for t, u in ((c.dqkv, c.o), (dqkv, o))]
    for n in both[0]:
        assert np.all(np.abs(both[0][n] - both[1][n]) <= 2 * (1.02 * r["err_" + n] + slack)), n


@pytest.mark.parametrize("where", ["q", "k", "v", "do"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("d,W", [(64, 0), (128, 90)])
def test_what_is_not_finite_stays_in_its_sequence(where, bad, d, W):
    """... and, of kv head 0, in its heads; as k, before it, in what sees it."""
    import torch
    banner(f"packed {bad} in {where} d={d} W={W}")
    lens, nh, nkv = [70, 130, 200, 1, 60], 4, 2
    off = offsets_of(lens, 0)
    T, hq = int(off[-1]), nh * d
    qkv = torch.randn((T, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((T, hq), device="cuda").to(torch.bfloat16)
    clean = Call(off, T, 200, nh, nkv, d, W, qkv.clone(), do.clone()).run()
    row = 150                                       # token 80 of the second sequence
    if where == "do":
        do[row, 3] = bad
    else:
        qkv[row, {"q": 0, "k": hq, "v": hq + nkv * d}[where] + 3] = bad
    c = Call(off, T, 200, nh, nkv, d, W, qkv, do).run()
    torch.cuda.synchronize()
    same = [host_f64(a) == host_f64(b) for a, b in zip(c.results(), clean.results())]
    others = np.ones(T, bool)
    others[70:200] = False
    assert same[0][others].all() and same[1][:, others].all() and same[2][others].all()
    # the other kv head's group
    assert same[0][:, hq // 2:].all() and same[1][2:].all()
    g = same[2].reshape(T, nh + 2 * nkv, d)
    assert g[:, 2:nh].all() and g[:, nh + 1].all() and g[:, nh + 3].all()
    if where == "k":
        assert same[0][70:150].all() and same[1][:, 70:150].all()


@pytest.mark.parametrize("nh,nkv,d", [(32, 8, 64), (64, 16, 64), (32, 8, 128)])
def test_what_is_not_finite_among_many_sequences(nh, nkv, d):
    """The same where blocks are many: each of four sequences has a NaN somewhere, the others
    keep their bits, and of the four every kv head's group but the first."""
    import torch
    banner(f"packed NaN among many {nh}/{nkv}x{d}")
    lens = [70, 130, 200, 1, 60] * 20
    off = offsets_of(lens, 0)
    T, hq = int(off[-1]), nh * d
    qkv = torch.randn((T, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((T, hq), device="cuda").to(torch.bfloat16)
    clean = Call(off, T, 200, nh, nkv, d, 0, qkv.clone(), do.clone(), fill=0.0).run()
    others = np.ones(T, bool)
    for i, (buf, col) in enumerate([(qkv, 0), (qkv, hq), (qkv, hq + nkv * d), (do, 0)]):
        s = 5 * i + 1                               # of 130 tokens
        buf[int(off[s]) + 80, col + 3] = float("nan")
        others[off[s]:off[s + 1]] = False
    c = Call(off, T, 200, nh, nkv, d, 0, qkv, do, fill=0.0).run()
    torch.cuda.synchronize()
    o, lse, g = [(a == b).cpu().numpy() for a, b in zip(c.results(), clean.results())]
    assert o[others].all() and lse[:, others].all() and g[others].all()
    grp = nh // nkv
    assert o[:, grp * d:].all() and lse[grp:].all()
    g = g.reshape(T, nh + 2 * nkv, d)
    assert g[:, grp:nh].all() and g[:, nh + 1:nh + nkv].all() and g[:, nh + nkv + 1:].all()
    assert not o.all() and not g.all()


def test_a_plan_of_other_sizes_writes_nothing():
    import torch
    banner("packed plan of other sizes")
    nh, nkv, d, T = 4, 2, 64, 300
    qkv = torch.randn((T, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((T, nh * d), device="cuda").to(torch.bfloat16)
    base = dict(off=[0, 100, 300], tokens=T, max_seq=200, window=0)
    for other in (dict(tokens=T + 64), dict(max_seq=199), dict(window=100),
                  dict(off=[0, 50, 100, 300])):
        c = Call(**dict(base), nh=nh, nkv=nkv, d=d, qkv=qkv, do=do, fill=3.0)
        o = Call(**dict(base, **other), nh=nh, nkv=nkv, d=d, qkv=qkv)
        o.L.forge_attention_packed_plan(o.cfg, o.off, o.plan, o.pos)
        n = min(o.plan.numel(), c.plan.numel())
        c.plan[:n] = o.plan[:n]
        c.run(plan=False)
        torch.cuda.synchronize()
        assert all(bool((t == 3.0).all()) for t in c.results()), other


def test_heads_may_differ_from_the_plan_s():
    import torch
    banner("packed plan for other heads")
    lens = [300, 5, 77]
    off = offsets_of(lens, 0)
    T = int(off[-1])
    a = Call(off, T, 300, 4, 2, 64, 0, torch.randn((T, 8 * 64), device="cuda").to(torch.bfloat16))
    b = Call(off, T, 300, 6, 3, 128, 0,
             torch.randn((T, 12 * 128), device="cuda").to(torch.bfloat16))
    a.run()
    b.run()
    want = b.o.clone()
    b.plan.copy_(a.plan)
    b.o.zero_()
    b.run(plan=False)
    torch.cuda.synchronize()
    assert torch.equal(b.o, want)


def test_replayed_from_a_graph_with_other_offsets():
    """Captured once; replays with other documents in the same bounds give the eager bits."""
    import torch
    banner("packed graph")
    nh, nkv, d, T = 4, 2, 128, 900
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    qkv = torch.randn((T, (nh + 2 * nkv) * d), device="cuda", generator=g).to(torch.bfloat16)
    do = torch.randn((T, nh * d), device="cuda", generator=g).to(torch.bfloat16)
    batches = [[0, 300, 900, 900, 900], [0, 1, 65, 500, 800], [10, 200, 264, 328, 900],
               [0, 0, 0, 0, 0]]
    c = Call(batches[0], T, 640, nh, nkv, d, 0, qkv, do, fill=3.0).run()
    e = Call(batches[0], T, 640, nh, nkv, d, 0, qkv, do, fill=3.0)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        c.run()
    for k in (1, 2, 3, 0, 1):
        for x in (c, e):
            x.off.copy_(torch.tensor(batches[k], dtype=torch.int32))
            for t in x.results():
                t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        e.run()
        torch.cuda.synchronize()
        for a, b in zip(c.results(), e.results()):
            assert torch.equal(a, b), k


def test_two_streams_at_once_and_again():
    """Each call has its own buffers: the bits of a run alone, every time."""
    import torch
    banner("packed on two streams")
    made = []
    for lens, nh, nkv, d in (([333, 1, 0, 200, 77], 6, 2, 64), ([700, 3, 400], 8, 2, 128)):
        off = offsets_of(lens, 0)
        T = int(off[-1])
        qkv = torch.randn((T, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
        do = torch.randn((T, nh * d), device="cuda").to(torch.bfloat16)
        made.append(Call(off, T, max(lens), nh, nkv, d, 0, qkv, do))
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    want = []
    for c, s in zip(made, streams):
        c.run(s)
        torch.cuda.synchronize()
        want.append([t.clone() for t in c.results()])
    for _ in range(3):
        for c, s in zip(made, streams):
            c.run(s)
    torch.cuda.synchronize()
    for c, w in zip(made, want):
        assert all(torch.equal(a, b) for a, b in zip(c.results(), w))


def test_many_sequences_and_far_rows():
    """More sequences than the plan's workgroup has threads, and rows whose elements lie
    beyond 2^31 bytes of the buffer: some sequences against their own few keys."""
    import torch
    from paper_2609_13645_amd import _lib
    banner("packed many sequences, far rows")
    nh, nkv, d = 32, 32, 128
    lens = [(7 * i) % 61 for i in range(5000)]
    off = offsets_of(lens, 0)
    T = int(off[-1])
    assert T * 3 * nh * d > 2 ** 30
    qkv = torch.empty((T, 3 * nh * d), dtype=torch.bfloat16, device="cuda").normal_()
    c = Call(off, T, 60, nh, nkv, d, 0, qkv, fill=0.0).run()
    torch.cuda.synchronize()
    x = qkv.view(T, 3, nh, d)
    for s in (0, 1, 8, 1023, 1024, 2500, 4999):
        a, n = int(off[s]), lens[s]
        if n == 0:
            continue
        q, k, v = (x[a:a + n, i].double().transpose(0, 1).contiguous() for i in range(3))
        z = (q @ k.transpose(1, 2).contiguous()) * d ** -0.5
        z = z.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), float("-inf"))
        assert float((c.lse[:, a:a + n].double() - z.logsumexp(2)).abs().max()) <= 1e-5
        o = (z.softmax(2) @ v).transpose(0, 1).reshape(n, nh * d)
        got = c.o[a:a + n].double()
        assert float((got - o).norm() / o.norm()) <= 2.0 ** -7


@pytest.mark.parametrize("more", [30, 600, 1500])
@pytest.mark.parametrize("longest", [2100, 131100])
def test_plans_of_every_size(more, longest):
    """Sequences few or more than a workgroup's threads, of few tiles or of more than its
    LDS has counts for: every row once, at its place (zero scores: its log-sum-exp is the
    log of its keys, whose number fp32 holds)."""
    import torch
    banner(f"packed plan more={more} longest={longest}")
    lens = [300, 0, longest, 65, 64, 1, 1900] + [(5 * i) % 97 for i in range(more)]
    off = offsets_of(lens, 3)
    T = int(off[-1]) + 7
    qkv = torch.zeros((T, 3 * 64), dtype=torch.bfloat16, device="cuda")
    c = Call(off, T, longest, 1, 1, 64, 0, qkv, fill=-9.0)
    for _ in range(2):
        c.pos.fill_(-7)
        c.lse.fill_(-9.0)
        c.run()
        torch.cuda.synchronize()
        pos = packed.positions(off, T, longest)
        inside = packed.covered(off, T, longest)
        assert np.array_equal(c.pos.cpu().numpy(), np.where(inside, pos, -7))
        lse = c.lse[0].cpu().numpy()
        assert np.all(lse[~inside] == -9.0)
        assert np.max(np.abs(lse[inside] - np.log(pos[inside] + 1.0))) <= 1e-5


@pytest.mark.parametrize("lens,n_seqs,max_seq,nh,nkv,d,W", [
    ([641], 1, 641, 4, 2, 64, 0), ([33] * 5 + [1, 1], 7, 33, 4, 2, 64, 0),
    ([1] * 7, 7, 1, 4, 1, 128, 0), ([320, 320, 58, 1, 1], 5, 320, 8, 2, 128, 0),
    ([1500], 1, 1500, 4, 2, 128, 66), ([2100, 2100, 33], 3, 2100, 16, 8, 64, 0)])
def test_workspace_at_the_lengths_that_need_most(lens, n_seqs, max_seq, nh, nkv, d, W):
    """... or all but a block for each sequence: nothing is written behind it, and the gradients
    are those that a workspace with room behind gives."""
    import torch
    banner(f"packed workspace {lens[:5]} d={d} W={W}")
    off = offsets_of(lens, 0)
    T = int(off[-1])
    qkv = torch.randn((T, (nh + 2 * nkv) * d), device="cuda").to(torch.bfloat16)
    do = torch.randn((T, nh * d), device="cuda").to(torch.bfloat16)
    c = Call(off, T, max_seq, nh, nkv, d, W, qkv, do, fill=3.0).run()
    want = c.dqkv.clone()
    n = c.ws.numel()
    room = torch.full((n + 65536,), 5.0, device="cuda")
    c.ws = room[:n]
    c.dqkv.fill_(3.0)
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.dqkv, want) and not bool(want.isnan().any())
    assert bool((room[n:] == 5.0).all())
