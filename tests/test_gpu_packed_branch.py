"""The operators of training on packed documents together, as a step of an attention branch
uses them: plan and positions, qkv product, rotation of a part of each head, packed attention,
output product, all of it backward, and one AdamW step of the branch's tensors with moments in
8 bits. Against the fp64 oracle; replayed from a graph with other documents in every replay;
and two branches on streams of their own at once."""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import packed
from gpu_util import rel_fro, dev_bf16, host_f64, banner

pytestmark = pytest.mark.gpu

B1, B2 = 0.9, 0.95
ROPE = dict(scaling="parts", factor=8.0, low_turns=1.0, high_turns=32.0, original_positions=256,
            amplitude=1.1)
SHAPES = [
    # lens, rows behind, hidden, heads, kv heads, head_dim, rot, offset, interleaved, window
    ([130, 0, 1, 257, 65], 9, 256, 4, 2, 64, 32, 32, True, 0),
    ([300, 41, 517], 0, 520, 6, 2, 128, 128, 0, False, 130),
]


class Branch:
    def __init__(self, shape, seed, stream=None):
        import torch
        from paper_2609_13645_amd import _lib
        self.L, self.stream, self.shape = _lib, stream, shape
        lens, behind, h, nh, nkv, d, rot, offset, inter, W = shape
        self.off_h = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.T, self.hq, self.width = int(self.off_h[-1]) + behind, nh * d, (nh + 2 * nkv) * d
        self.n_pos, self.n_rot = max(lens), nh + nkv
        rng = np.random.default_rng(seed)

        def bits(shape, std):
            return fi.to_bf16_bits((std * rng.standard_normal(shape)).astype(np.float32))
        b = dict(x=bits((self.T, h), 1.0), w_qkv=bits((self.width, h), h ** -0.5),
                 w_o=bits((h, self.hq), self.hq ** -0.5), dy=bits((self.T, h), 1.0))
        self.ref = {n: fi.bf16_bits_to_f64(v) for n, v in b.items()}
        self.i = {n: dev_bf16(v) for n, v in b.items()}
        e = lambda *s, dt=torch.bfloat16: torch.full(s, float("nan"), dtype=dt, device="cuda")
        f = torch.float32
        # (rows behind the last document: attention leaves them as they are, so they are zeros)
        z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        self.o = dict(qkv=e(self.T, self.width), att=z(self.T, self.hq), lse=e(nh, self.T, dt=f),
                      y=e(self.T, h), datt=e(self.T, self.hq), dqkv=z(self.T, self.width),
                      dx=e(self.T, h), dw_qkv=e(self.width, h, dt=f), dw_o=e(h, self.hq, dt=f))
        self.off = torch.from_numpy(self.off_h).cuda()
        self.pos = torch.zeros(self.T, dtype=torch.int32, device="cuda")
        self.rope = _lib.rope_part_cfg(dict(head_dim=d, rot_dim=rot, rot_offset=offset,
                                            interleaved=inter, **ROPE))
        self.attn = _lib.attn_packed_cfg(dict(tokens=self.T, n_seqs=len(lens), max_seq=self.T,
                                              n_heads=nh, n_kv_heads=nkv, head_dim=d, window=W))
        byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        self.plan = byte(_lib.forge_attention_packed_plan_bytes(self.attn))
        self.ws = byte(_lib.forge_attention_packed_bwd_workspace_bytes(self.attn))
        self.cos, self.sin = (torch.empty((self.n_pos, rot // 2), device="cuda") for _ in range(2))
        _lib.forge_rope_part_table(self.rope, None, self.n_pos, 1e4, self.cos, self.sin)
        self.state = {}
        for k, n in enumerate(("w_qkv", "w_o")):
            w = self.i[n]
            blocks = -(-w.numel() // _lib.ADAMW_BLOCK)
            self.state[n] = dict(
                master=w.float().view(-1), param=w, grad=self.o["d" + n], lr_scale=(1.0, 0.5)[k],
                m=torch.zeros(w.numel(), dtype=torch.int8, device="cuda"),
                v=torch.zeros(w.numel(), dtype=torch.uint8, device="cuda"),
                m_scale=torch.zeros(blocks, device="cuda"), v_scale=torch.zeros(blocks, device="cuda"))
        self.tensors = _lib.adamw_multi_tensors(list(self.state.values()))
        self.scalars = torch.tensor([1e-3, 1.0, 1.0, 1.0], device="cuda")
        self.step = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.values = {n: e(w["m"].numel()) for n, w in self.state.items()}

    def run(self):
        L, i, o, T, s = self.L, self.i, self.o, self.T, self.stream
        h, hq, w, KC, MC = self.shape[2], self.hq, self.width, self.L.GEMM_KC, self.L.GEMM_MC
        rot = (w, self.cos, self.sin, self.pos, T, self.n_pos, self.n_rot)
        L.forge_attention_packed_plan(self.attn, self.off, self.plan, self.pos, s)
        L.forge_gemm(KC, KC, L.EPI_STORE_BF16, i["x"], i["w_qkv"], o["qkv"], None, T, w, h, h, h, w,
                     0, s)
        L.forge_rope_part_apply(self.rope, o["qkv"], w, o["qkv"], *rot, False, s)
        L.forge_attention_packed_fwd(self.attn, self.plan, o["qkv"], o["att"], o["lse"], s)
        L.forge_gemm(KC, KC, L.EPI_RESID_BF16, o["att"], i["w_o"], o["y"], i["x"], T, h, hq, hq,
                     hq, h, h, s)
        L.forge_gemm(KC, MC, L.EPI_STORE_BF16, i["dy"], i["w_o"], o["datt"], None, T, hq, h, h, hq,
                     hq, 0, s)
        L.forge_gemm(MC, MC, L.EPI_STORE_F32, i["dy"], o["att"], o["dw_o"], None, h, hq, T, h, hq,
                     hq, 0, s)
        L.forge_attention_packed_bwd(self.attn, self.plan, o["qkv"], o["att"], o["lse"], o["datt"],
                                     o["dqkv"], self.ws, s)
        L.forge_rope_part_apply(self.rope, o["dqkv"], w, o["dqkv"], *rot, True, s)
        L.forge_gemm(KC, MC, L.EPI_STORE_BF16, o["dqkv"], i["w_qkv"], o["dx"], None, T, h, w, w, h,
                     h, 0, s)
        L.forge_gemm(MC, MC, L.EPI_STORE_F32, o["dqkv"], i["x"], o["dw_qkv"], None, w, h, T, w, h,
                     h, 0, s)
        L.forge_adamw_advance(self.scalars, self.step, 1e-3, B1, B2, s)
        L.forge_adamw_multi_step(self.tensors, 8, False, L.AdamwHparams(B1, B2, 1e-8, 0.1),
                                 self.scalars, self.step, s)
        L.forge_adamw_multi_read(self.tensors, L.pointers(list(self.values.values())), None, True, s)

    def results(self):
        r = {n: t for n, t in self.o.items() if n != "lse"}
        for n, w in self.state.items():
            r.update({f"{n}.{k}": t for k, t in w.items() if k not in ("grad", "lr_scale")})
            r[n + ".values"] = self.values[n]
        return dict(r, pos=self.pos)

    def oracle(self):
        lens, behind, h, nh, nkv, d, rot, offset, inter, W = self.shape
        r, T, hq, k0 = self.ref, self.T, self.hq, (nh + nkv) * d
        inside = packed.covered(self.off_h, T, T)
        pos = np.maximum(packed.positions(self.off_h, T, T), 0)
        w = packed.part_frequencies(rot, 1e4, "parts", 8.0, 1.0, 32.0, 256)

        def turn(x, backward=False):
            y = x.copy()
            y[:, :k0] = packed.rope_part(x[:, :k0].reshape(T, nh + nkv, d), pos, rot, offset, inter,
                                         w, 1.1, backward).reshape(T, k0)
            return y
        qkv = turn(r["x"] @ r["w_qkv"].T)
        datt = r["dy"] @ r["w_o"]
        t = packed.attention(qkv[:, :hq].reshape(T, nh, d), qkv[:, hq:k0].reshape(T, nkv, d),
                             qkv[:, k0:].reshape(T, nkv, d), datt.reshape(T, nh, d), self.off_h, T, W)
        rows = lambda x: np.where(inside[:, None], x.reshape(T, -1), 0.0)
        att = rows(t["o"])
        dqkv = turn(np.concatenate([rows(t[n]) for n in ("dq", "dk", "dv")], axis=1), True)
        return dict(y=r["x"] + att @ r["w_o"].T, dx=dqkv @ r["w_qkv"], dw_qkv=dqkv.T @ r["x"],
                    dw_o=r["dy"].T @ att)


@pytest.mark.parametrize("shape", SHAPES)
def test_step_of_a_branch(shape):
    """Six roundings to bf16 one behind another on the longest way (product, rotation,
    probabilities, score gradient, attention's gradients, rotation back): 6 2^-8, each a
    relative error of the whole that the steps between pass on about as it is. The optimizer,
    from the gradients that it was given: the oracle's codes; values within a bf16 rounding
    of the decoded ones."""
    import torch
    banner(f"packed branch {shape}")
    b = Branch(shape, 21)
    before = {n: w["master"].double().cpu().numpy() for n, w in b.state.items()}
    b.run()
    torch.cuda.synchronize()
    for n, ref in b.oracle().items():
        assert rel_fro(host_f64(b.o[n]), ref) <= 6 * 2.0 ** -8, n
    lr, c1, c2, _ = (float(x) for x in b.scalars.cpu())
    for k, (n, w) in enumerate(b.state.items()):
        g = w["grad"].cpu().numpy().reshape(-1)
        zero = np.zeros(g.size, np.float32)
        scale = np.zeros(w["m_scale"].numel(), np.float32)
        m, v = packed.moments_step(g, zero.astype(np.int8), scale, zero.astype(np.uint8), scale, B1,
                                   B2, 1.0)
        u = packed.moment_draws(g.size, k, 1)
        for name, (q, s) in dict(m=packed.encode_m(m, u[0]), v=packed.encode_v(v, u[1])).items():
            assert np.array_equal(w[name].cpu().numpy(), q), (n, name)
            assert np.array_equal(w[name + "_scale"].cpu().numpy(), s), (n, name)
            if name == "m":
                kept = packed.decode_m(q, s).astype(np.float64)
                assert np.all(np.abs(host_f64(b.values[n]) - kept) <= 2.0 ** -8 * np.abs(kept))
        p0, m, v = before[n], m.astype(np.float64), v.astype(np.float64)
        wd, eps = (float(np.float32(x)) for x in (0.1, 1e-8))
        p = p0 - lr * w["lr_scale"] * (m / c1 / (np.sqrt(v / c2) + eps) + wd * p0)
        got = host_f64(w["master"])
        slack = 2.0 ** -24 * np.linalg.norm(p0)
        assert np.linalg.norm(got - p) <= 1e-5 * np.linalg.norm(p - p0) + slack, n
        assert np.all(np.abs(host_f64(w["param"]).reshape(-1) - got) <= 2.0 ** -8 * np.abs(got))


def test_steps_replayed_from_a_graph():
    """Captured once, replayed with other documents each time and eager steps in between: the
    bits of eager steps."""
    import torch
    banner("packed branch graph")
    a, b = Branch(SHAPES[0], 1), Branch(SHAPES[0], 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        a.run()
    last = int(a.off_h[-1])
    batches = [a.off_h, [0, 1, 64, 129, 130, last], [0, 0, 200, 201, last, last],
               [0, 128, 256, 256, 300, last], [0, last, last, last, last, last]]
    for k, off in enumerate(batches):
        for x in (a, b):
            x.off.copy_(torch.tensor(np.asarray(off), dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        b.run()
        torch.cuda.synchronize()
        for (n, t), w in zip(a.results().items(), b.results().values()):
            assert torch.equal(t, w), (k, n)


def test_two_branches_at_once():
    """Steps on two streams side by side: the bits of steps taken alone."""
    import torch
    banner("packed branches on two streams")
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    alone, both = ([Branch(s, 5 + k, streams[k]) for k, s in enumerate(SHAPES)] for _ in range(2))
    torch.cuda.synchronize()
    for b in alone:
        for _ in range(3):
            b.run()
        torch.cuda.synchronize()
    for _ in range(3):
        for b in both:
            b.run()
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        for (n, t), w in zip(x.results().items(), y.results().values()):
            assert torch.equal(t, w), n
