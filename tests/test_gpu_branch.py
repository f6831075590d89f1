"""LayerNorm, rotary axes and window attention together, as an attention branch
uses them: norm, qkv product, rotation, attention, output product with the
residual, and all of it backward, against the fp64 oracle; replayed from a
captured graph; and on a stream of its own."""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import branch
from gpu_util import rel_fro, host_f64, banner

pytestmark = pytest.mark.gpu

EPS = 1e-5
SHAPES = [
    # batch, seq, hidden, heads, kv heads, head_dim, pairs, window, sinks, lens
    (2, 200, 256, 4, 2, 64, (8, 12, 12), 64, 4, (200, 133)),
    (1, 517, 520, 6, 2, 128, (16, 24, 24), 130, 0, None),
]


class Branch:
    """The branch's device buffers and its calls, forward and backward."""

    def __init__(self, shape, seed, stream=None):
        import torch
        from paper_2609_13645_amd import _lib
        self.L, self.stream = _lib, stream
        B, S, h, nh, nkv, d, pairs, W, sinks, lens = self.shape = shape
        self.T, self.hq, self.width = B * S, nh * d, (nh + 2 * nkv) * d
        self.n_rot = nh + nkv
        rng = np.random.default_rng(seed)

        def bits(shape, std, mean=0.0):
            return fi.to_bf16_bits((mean + std * rng.standard_normal(shape)).astype(np.float32))
        b = dict(x=bits((self.T, h), 1.0), g=bits(h, 0.2, 1.0), b=bits(h, 0.2),
                 w_qkv=bits((self.width, h), h ** -0.5), w_o=bits((h, self.hq), self.hq ** -0.5),
                 dy=bits((self.T, h), 1.0))
        self.ref = {n: fi.bf16_bits_to_f64(v) for n, v in b.items()}
        from gpu_util import dev_bf16
        self.i = {n: dev_bf16(v) for n, v in b.items()}
        self.pos_h = rng.integers(0, 50, (len(pairs), self.T)).astype(np.int32)
        self.pos = torch.from_numpy(self.pos_h).cuda()
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.rope = _lib.rope_axes_cfg(dict(head_dim=d, pairs=pairs))
        self.attn = _lib.AttnWindowCfg(B, S, nh, nkv, d, W, sinks)
        e = lambda *s, dt=torch.bfloat16: torch.full(s, float("nan"), dtype=dt, device="cuda")
        f = torch.float32
        self.o = dict(
            a=e(self.T, h), mean=e(self.T, dt=f), rstd=e(self.T, dt=f), qkv=e(self.T, self.width),
            att=e(self.T, self.hq), lse=e(B, nh, S, dt=f), y=e(self.T, h), datt=e(self.T, self.hq),
            dqkv=e(self.T, self.width), da=e(self.T, h), dx=e(self.T, h), dg=e(h, dt=f),
            db=e(h, dt=f), dw_qkv=e(self.width, h, dt=f), dw_o=e(h, self.hq, dt=f))
        self.cos, self.sin = (torch.empty((50, d // 2), device="cuda") for _ in range(2))
        _lib.forge_rope_axes_table(self.rope, 50, 1e4, self.cos, self.sin)
        ws = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
        self.ws = ws(_lib.forge_attention_window_bwd_workspace_bytes(self.attn))
        self.nws = ws(_lib.forge_layernorm_bwd_workspace_bytes(self.T, h))

    def run(self):
        L, i, o, T, h, s = self.L, self.i, self.o, self.T, self.shape[2], self.stream
        hq, w, KC, MC = self.hq, self.width, self.L.GEMM_KC, self.L.GEMM_MC
        rot = (w, self.cos, self.sin, self.pos, T, 50, self.n_rot)
        L.forge_layernorm_fwd(i["x"], i["g"], i["b"], o["a"], o["mean"], o["rstd"], T, h, EPS, s)
        L.forge_gemm(KC, KC, L.EPI_STORE_BF16, o["a"], i["w_qkv"], o["qkv"], None, T, w, h, h, h, w,
                     0, s)
        L.forge_rope_axes_apply(self.rope, o["qkv"], w, o["qkv"], *rot, False, s)
        L.forge_attention_window_fwd(self.attn, o["qkv"], self.lens, o["att"], o["lse"], s)
        L.forge_gemm(KC, KC, L.EPI_RESID_BF16, o["att"], i["w_o"], o["y"], i["x"], T, h, hq, hq,
                     hq, h, h, s)
        L.forge_gemm(KC, MC, L.EPI_STORE_BF16, i["dy"], i["w_o"], o["datt"], None, T, hq, h, h, hq,
                     hq, 0, s)
        L.forge_gemm(MC, MC, L.EPI_STORE_F32, i["dy"], o["att"], o["dw_o"], None, h, hq, T, h, hq,
                     hq, 0, s)
        L.forge_attention_window_bwd(self.attn, o["qkv"], self.lens, o["att"], o["lse"], o["datt"],
                                     o["dqkv"], self.ws, s)
        L.forge_rope_axes_apply(self.rope, o["dqkv"], w, o["dqkv"], *rot, True, s)
        L.forge_gemm(KC, MC, L.EPI_STORE_BF16, o["dqkv"], i["w_qkv"], o["da"], None, T, h, w, w, h,
                     h, 0, s)
        L.forge_gemm(MC, MC, L.EPI_STORE_F32, o["dqkv"], o["a"], o["dw_qkv"], None, w, h, T, w, h,
                     h, 0, s)
        L.forge_layernorm_bwd(i["x"], i["g"], o["mean"], o["rstd"], o["da"], i["dy"], o["dx"],
                              o["dg"], o["db"], False, T, h, self.nws, s)

    RESULTS = ("y", "dx", "dg", "db", "dw_qkv", "dw_o")

    def oracle(self):
        B, S, h, nh, nkv, d, pairs, W, sinks, lens = self.shape
        r, T, hq, k0 = self.ref, self.T, self.hq, (nh + nkv) * d

        def turn(x, inverse=False):
            y = x.copy()
            y[:, :k0] = branch.rope_axes(x[:, :k0].reshape(T, nh + nkv, d), self.pos_h, pairs,
                                         False, False, 1e4, inverse).reshape(T, k0)
            return y
        a, m, rs = branch.layernorm_fwd(r["x"], r["g"], r["b"], EPS)
        qkv = turn(a @ r["w_qkv"].T)
        datt = r["dy"] @ r["w_o"]
        t = branch.window_attention(qkv[:, :hq].reshape(T, nh, d), qkv[:, hq:k0].reshape(T, nkv, d),
                                    qkv[:, k0:].reshape(T, nkv, d), datt.reshape(T, nh, d), B, S, W,
                                    sinks, lens)
        att = t["o"].reshape(T, hq)
        dqkv = turn(np.concatenate([t[n].reshape(T, -1) for n in ("dq", "dk", "dv")], axis=1), True)
        dx, dg, db = branch.layernorm_bwd(r["x"], r["g"], m, rs, dqkv @ r["w_qkv"])
        return dict(y=r["x"] + att @ r["w_o"].T, dx=dx + r["dy"], dg=dg, db=db, dw_qkv=dqkv.T @ a,
                    dw_o=r["dy"].T @ att)


@pytest.mark.parametrize("shape", SHAPES)
def test_branch_forward_and_backward(shape):
    """Six roundings to bf16 one behind another on the longest way (norm, product,
    rotation, attention with its probabilities, product): 6 2^-8, each a relative
    error of the whole that the steps between pass on about as it is."""
    import torch
    banner(f"branch {shape}")
    b = Branch(shape, 11)
    b.run()
    torch.cuda.synchronize()
    for n, ref in b.oracle().items():
        assert rel_fro(host_f64(b.o[n]), ref) <= 6 * 2.0 ** -8, n


def test_branch_replayed_from_a_graph():
    """Captured once, replayed with new inputs and eager runs in between: each replay
    gives the eager bits."""
    import torch
    banner("branch graph")
    b, other = Branch(SHAPES[0], 1), Branch(SHAPES[0], 2)
    side = torch.cuda.Stream()
    b.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        b.run()
    for k in range(4):
        for t in b.o.values():
            t.fill_(float("nan"))
        b.i["x"].copy_(other.i["x"] if k % 2 else b.i["x"].flip(0))
        g.replay()
        torch.cuda.synchronize()
        got = {n: b.o[n].clone() for n in b.o}
        other.run()
        b.run()
        torch.cuda.synchronize()
        for n in b.o:
            assert torch.equal(got[n], b.o[n]), (k, n)


def test_branch_on_another_stream_beside_the_current_one():
    """Two branches on two streams at once: each has its own buffers and the bits of
    a run alone."""
    import torch
    banner("branch on two streams")
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = Branch(SHAPES[0], 5, s1), Branch(SHAPES[1], 6, s2)
    torch.cuda.synchronize()
    want = []
    for x in (a, b):
        x.run()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in x.o.items()})
    for _ in range(3):
        for x in (a, b):
            x.run()
    torch.cuda.synchronize()
    for x, w in zip((a, b), want):
        for n, t in x.o.items():
            assert torch.equal(t, w[n]), n
