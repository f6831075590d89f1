"""forge_adamw_multi_step / _read on the GPU: with moments in 32 bits the bits of
forge_adamw_step; in 8 bits the oracle's codes and scales, all of them, and a master
update within 1e-5 of the fp64 one of the same moments (relative Frobenius, as the
plain step's)."""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import adamw as oadam, packed
from gpu_util import rel_fro, banner

pytestmark = pytest.mark.gpu

B1, B2, EPS, WD, LR = 0.9, 0.95, 1e-8, 0.1, 1e-3
SIZES = [[1], [255, 256, 257], [4096, 0, 1000, 1, 70001], [300 + 7 * i for i in range(67)],
         [1 << 20, 5, 333333]]


def f32(x):
    return float(np.float32(x))


class Tensors:
    """Host state of a list of tensors, and the same on the GPU behind guard bytes."""

    GUARD = 64

    def __init__(self, sizes, bits, bf16_grads, seed, step=3):
        import torch
        rng = np.random.default_rng(seed)
        self.bits, self.bf16, self.step, self.host, self.dev, self.raw = bits, bf16_grads, step, [], [], []
        for k, n in enumerate(sizes):
            h = dict(master=(0.02 * rng.standard_normal(n)).astype(np.float32),
                     grad=(1e-3 * rng.standard_normal(n)).astype(np.float32))
            if n > 600:
                h["grad"][256:512] = 0.0                       # a block without gradients
            if bf16_grads:
                h["grad_bits"] = fi.to_bf16_bits(h["grad"])
                h["grad"] = fi.bf16_bits_to_f64(h["grad_bits"]).astype(np.float32)
            m = (3e-4 * rng.standard_normal(n)).astype(np.float32)
            v = (1e-6 * (0.05 + rng.random(n)) ** 2).astype(np.float32)
            if n > 600:
                m[256:512] = v[256:512] = 0.0
            if bits == 8 and n:
                half = np.full(n, np.float32(0.5))
                h["m"], h["m_scale"] = packed.encode_m(m, half)
                h["v"], h["v_scale"] = packed.encode_v(v, half)
            else:
                h["m"], h["v"] = m, v
            h["lr_scale"], h["decay_scale"] = (1.0, 0.5, 2.0)[k % 3], (1.0, 0.0)[k % 2]
            self.host.append(h)
            d = dict(n=n, lr_scale=h["lr_scale"], decay_scale=h["decay_scale"])
            for name in ("master", "grad", "m", "v", "m_scale", "v_scale"):
                if name in h:
                    x = h["grad_bits"] if name == "grad" and bf16_grads else h[name]
                    d[name] = self._guarded(torch.from_numpy(np.ascontiguousarray(x)))
            d["param"] = self._guarded(torch.zeros(n, dtype=torch.bfloat16))
            self.dev.append(d)
        self.scalars = torch.tensor([LR, 1 - B1 ** step, 1 - B2 ** step, 0.7], device="cuda")

    def _guarded(self, x):
        """x on the GPU, bytes of 0xA5 before and behind it."""
        import torch
        raw = torch.full((x.numel() * x.element_size() + 2 * self.GUARD,), 0xA5, dtype=torch.uint8,
                         device="cuda")
        self.raw.append(raw)
        mid = raw[self.GUARD:raw.numel() - self.GUARD]
        mid.copy_(x.reshape(-1).view(torch.uint8)) if x.numel() else None
        return mid.view(x.dtype) if x.numel() else mid

    def check_guards(self):
        for r in self.raw:
            g = self.GUARD
            assert bool((r[:g] == 0xA5).all()) and bool((r[r.numel() - g:] == 0xA5).all())

    def call(self, seed=None, stream=None):
        from paper_2609_13645_amd import _lib
        hp = _lib.AdamwHparams(B1, B2, EPS, WD)
        _lib.forge_adamw_multi_step(_lib.adamw_multi_tensors(self.dev), self.bits, self.bf16, hp,
                                    self.scalars, seed, stream)

    def got(self, k, name):
        x = self.dev[k][name].cpu()
        return x.view(__import__("torch").int16).numpy().view(np.uint16) if name == "param" \
            else x.numpy()


@pytest.mark.parametrize("sizes", SIZES)
def test_32_bits_are_the_plain_step_s(sizes):
    """Scales of 1 and fp32 gradients: bit for bit."""
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"adamw multi 32 {sizes[:5]}")
    t, one = Tensors(sizes, 32, False, 1), Tensors(sizes, 32, False, 1)
    for d in t.dev:
        d["lr_scale"] = d["decay_scale"] = 1.0
    t.call()
    hp = _lib.AdamwHparams(B1, B2, EPS, WD)
    for d in one.dev:
        _lib.forge_adamw_step(d["master"], d["param"], d["grad"], d["m"], d["v"], d["n"], hp,
                              one.scalars)
    torch.cuda.synchronize()
    t.check_guards()
    for k in range(len(sizes)):
        for name in ("master", "m", "v", "param"):
            assert np.array_equal(t.got(k, name), one.got(k, name)), (k, name)


def _reference(h, m, v, step):
    """The fp64 update of the new moments m and v."""
    bc1, bc2 = (f32(x) for x in oadam.bias_corrections(B1, B2, step))
    p, lr = h["master"].astype(np.float64), f32(LR) * h["lr_scale"]
    m, v = m.astype(np.float64), v.astype(np.float64)
    return p - lr * (m / bc1 / (np.sqrt(v / bc2) + f32(EPS)) + f32(WD) * h["decay_scale"] * p)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
def test_32_bits_with_scales(sizes, bf16):
    import torch
    banner(f"adamw multi 32 with scales {sizes[:5]} bf16={bf16}")
    t = Tensors(sizes, 32, bf16, 2)
    t.call()
    torch.cuda.synchronize()
    t.check_guards()
    for k, h in enumerate(t.host):
        if not sizes[k]:
            continue
        g = h["grad"].astype(np.float64) * f32(0.7)
        m = f32(B1) * h["m"].astype(np.float64) + (1 - f32(B1)) * g
        v = f32(B2) * h["v"].astype(np.float64) + (1 - f32(B2)) * g * g
        p, p0 = _reference(h, m, v, t.step), h["master"].astype(np.float64)
        # a new master is rounded to 2^-24 of itself, which of a tensor of one element is
        # more than 1e-5 of its step of 1e-3
        slack = 2.0 ** -24 * np.linalg.norm(p0)
        assert np.linalg.norm(t.got(k, "master") - p) <= 1e-5 * np.linalg.norm(p - p0) + slack, k
        assert rel_fro(t.got(k, "m"), m) <= 1e-6 and rel_fro(t.got(k, "v"), v) <= 1e-6
        assert np.array_equal(t.got(k, "param"), fi.to_bf16_bits(t.got(k, "master")))


@pytest.mark.parametrize("seed", [None, 12345, -1])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
def test_8_bits(sizes, bf16, seed):
    """Three steps one behind another, the codes of each those of the oracle."""
    import torch
    banner(f"adamw multi 8 {sizes[:5]} bf16={bf16} seed={seed}")
    t = Tensors(sizes, 8, bf16, 3)
    dev_seed = None if seed is None else torch.tensor([seed], dtype=torch.int32, device="cuda")
    for s in range(3):
        t.call(dev_seed)
        torch.cuda.synchronize()
        for k, h in enumerate(t.host):
            if not sizes[k]:
                continue
            m, v = packed.moments_step(h["grad"], h["m"], h["m_scale"], h["v"], h["v_scale"], B1,
                                       B2, 0.7)
            u = packed.moment_draws(sizes[k], k, None if seed is None else seed & 0xFFFFFFFF)
            p, p0 = _reference(h, m, v, t.step), h["master"].astype(np.float64)
            h["m"], h["m_scale"] = packed.encode_m(m, u[0])
            h["v"], h["v_scale"] = packed.encode_v(v, u[1])
            for name in ("m_scale", "v_scale", "m", "v"):
                assert np.array_equal(t.got(k, name), h[name]), (s, k, name)
            slack = 2.0 ** -24 * np.linalg.norm(p0)
            h["master"] = t.got(k, "master")
            assert np.linalg.norm(h["master"] - p) <= 1e-5 * np.linalg.norm(p - p0) + slack, (s, k)
            assert np.array_equal(t.got(k, "param"), fi.to_bf16_bits(h["master"]))
        if dev_seed is not None:
            dev_seed += 1
            seed += 1
    t.check_guards()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
def test_read(sizes, bf16):
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"adamw multi read {sizes[:5]} bf16={bf16}")
    t = Tensors(sizes, 8, False, 4)
    dt = torch.bfloat16 if bf16 else torch.float32
    out = [[t._guarded(torch.zeros(n, dtype=dt)) for n in sizes] for _ in range(2)]
    lst = _lib.adamw_multi_tensors(t.dev)
    m, v = (_lib.pointers(o) for o in out)
    for args, filled in (((m, None), (1, 0)), ((None, v), (0, 1)), ((m, v), (1, 1))):
        for o in out[0] + out[1]:
            o.zero_()
        _lib.forge_adamw_multi_read(lst, *args, bf16)
        torch.cuda.synchronize()
        for k, h in enumerate(t.host):
            for o, yes, dec, name in ((out[0], filled[0], packed.decode_m, "m"),
                                      (out[1], filled[1], packed.decode_v, "v")):
                if not sizes[k]:
                    continue
                want = dec(h[name], h[name + "_scale"]) if yes else np.zeros(sizes[k], np.float32)
                got = o[k].cpu()
                if bf16:
                    assert np.array_equal(got.view(torch.int16).numpy().view(np.uint16),
                                          fi.to_bf16_bits(want))
                else:
                    assert np.array_equal(got.numpy(), want)
    t.check_guards()


def test_what_is_not_finite_stays_in_its_block():
    import torch
    banner("adamw multi NaN")
    sizes = [2000, 700]
    for bad in (float("nan"), float("inf"), float("-inf")):
        t, fine = Tensors(sizes, 8, False, 5), Tensors(sizes, 8, False, 5)
        t.dev[0]["grad"][1030] = bad
        t.call()
        fine.call()
        torch.cuda.synchronize()
        for name in ("m_scale", "v_scale"):
            s = t.got(0, name)
            assert np.isnan(s[4]) and np.array_equal(np.delete(s, 4), np.delete(fine.got(0, name), 4))
            assert np.array_equal(t.got(1, name), fine.got(1, name))
        keep = np.arange(2000) // 256 != 4
        for name in ("m", "v"):
            assert np.array_equal(t.got(0, name)[keep], fine.got(0, name)[keep])
            assert not t.got(0, name)[~keep].any()
        p, q = t.got(0, "master"), fine.got(0, "master")
        assert np.isnan(p[1030]) and np.array_equal(np.delete(p, 1030), np.delete(q, 1030))


def test_tiny_and_untouched_blocks():
    """Blocks of zeros stay zeros; moments below 2^-94 are kept as zeros."""
    import torch
    banner("adamw multi tiny blocks")
    t = Tensors([1024], 8, False, 6)
    d = t.dev[0]
    for name in ("m", "v", "m_scale", "v_scale", "grad"):
        d[name].zero_()
    d["grad"][256:512] = 2.0 ** -92
    d["grad"][512:768] = 1e-25          # v underflows, m does not
    p0 = t.got(0, "master").copy()
    t.call()
    torch.cuda.synchronize()
    sm, sv = t.got(0, "m_scale"), t.got(0, "v_scale")
    assert sm[0] == sm[1] == sm[3] == 0 and sm[2] > 0 and not sv.any()
    assert not t.got(0, "v").any() and (t.got(0, "m")[512:768] == 127).all()
    decay = 1 - f32(LR) * f32(WD)
    assert np.allclose(t.got(0, "master"), p0 * decay, rtol=1e-6)


def test_a_step_captured_and_replayed():
    """The seed is the step counter on the device: each replay draws anew, and gives the
    eager run's bits."""
    import torch
    from paper_2609_13645_amd import _lib
    banner("adamw multi graph")
    sizes = [5000, 1, 300] * 15
    runs = [Tensors(sizes, 8, True, 7), Tensors(sizes, 8, True, 7)]
    steps = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in runs]
    side = torch.cuda.Stream()

    def one(t, n, stream=None):
        _lib.forge_adamw_advance(t.scalars, n, LR, B1, B2, stream)
        t.call(n, stream)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        one(runs[0], steps[0])
    for k in range(4):
        g.replay()
        torch.cuda.synchronize()
        one(runs[1], steps[1], side)
        side.synchronize()
        for i in range(len(sizes)):
            for name in ("master", "param", "m", "v", "m_scale", "v_scale"):
                assert np.array_equal(runs[0].got(i, name), runs[1].got(i, name)), (k, i, name)


def test_drawn_codes_follow_a_falling_gradient():
    """Gradients that fall to a tenth, beta2 0.999: drawn codes follow the 32-bit v in the
    mean; rounded to the nearest, a decay of 0.1 % a step would not move them within their
    block. A draw between codes q and q + 1, 4 / q of v apart, adds a variance of (4 / q)^2 / 6
    on average, of which the sum over 1 / (1 - beta2) steps with falling weights is (4 / q)^2 / 6
    / (2 * 0.001). Here q is 25 or more: 1.5 times v at most, and 1.5 / sqrt(4032) = 0.023 for the
    mean over the elements. Five of those: 0.12."""
    import torch
    from paper_2609_13645_amd import _lib
    banner("adamw multi falling gradient")
    n, hp = 4096, _lib.AdamwHparams(0.9, 0.999, 1e-8, 0.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    size = 10 ** torch.empty(n, device="cuda").uniform_(-1, 0, generator=g)
    # one element in 64 keeps its gradients: the blocks' scales do not fall with the others
    fall = torch.where(torch.arange(n, device="cuda") % 64 == 0, 1.0, 0.1)
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")
    f, grad = torch.float32, torch.zeros(n, device="cuda")
    a = dict(master=z(f), param=z(torch.bfloat16), grad=grad, m=z(f), v=z(f))
    b = dict(a, master=z(f), param=z(torch.bfloat16), m=z(torch.int8), v=z(torch.uint8),
             m_scale=z(f, 16), v_scale=z(f, 16))
    sc, step = torch.tensor([1e-4, 1, 1, 1.0], device="cuda"), z(torch.int32, 1)
    la, lb = _lib.adamw_multi_tensors([a]), _lib.adamw_multi_tensors([b])
    for k in range(4000):
        grad.normal_(generator=g).mul_(size if k < 1000 else size * fall)
        _lib.forge_adamw_advance(sc, step, 1e-4, 0.9, 0.999)
        _lib.forge_adamw_multi_step(la, 32, False, hp, sc)
        _lib.forge_adamw_multi_step(lb, 8, False, hp, sc, step)
    v = z(f)
    _lib.forge_adamw_multi_read(lb, None, _lib.pointers([v]))
    torch.cuda.synchronize()
    keep = fall < 1
    ratio = (v[keep].double() / a["v"][keep].double()).mean().item()
    assert abs(ratio - 1) <= 0.12, ratio


@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_moments_whose_v_is_lost(beta2):
    """Gradients below 2^-47, then none, with the smallest eps that 8 bits take: v of the first
    step, (1 - beta2) 2^-94 at most, is kept as zero, m is not. The second update is m' / eps where
    the 32-bit one is m / (r + eps), r = sqrt(v') below 2^-47 (bias-corrected: (beta2 (1 - beta2) /
    (1 - beta2^2))^(1/2) |g|, below 0.71 2^-47). So they differ by r / eps of themselves, below
    0.71 2^-7, and by m' - m, half a code at most: (2 * 127 + 1) / 2 / 127^2 of the largest |m|. Both steps
    also by the hardware's root and quotient, below 2^-20. With m-hat = 0.9 * 0.1 / 0.19 |g| below
    0.474 2^-47, and a first update below 2^-47 / 2^-40."""
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"adamw multi lost v beta2={beta2}")
    n, lr, eps = 3000, 1.0, _lib.ADAMW_MIN_EPS_8BIT
    hp = _lib.AdamwHparams(0.9, beta2, eps, 0.0)
    rng = np.random.default_rng(9)
    g = (2.0 ** -47 * (0.5 + 0.49 * rng.random(n)) * rng.choice([-1, 1], n)).astype(np.float32)
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")
    f = torch.float32
    runs = {}
    for bits in (32, 8):
        t = dict(master=z(f), param=z(torch.bfloat16), grad=torch.from_numpy(g).cuda())
        blocks = -(-n // _lib.ADAMW_BLOCK)
        t.update(dict(m=z(f), v=z(f)) if bits == 32 else dict(
            m=z(torch.int8), v=z(torch.uint8), m_scale=z(f, blocks), v_scale=z(f, blocks)))
        sc, step = torch.tensor([lr, 1, 1, 1.0], device="cuda"), z(torch.int32, 1)
        lst = _lib.adamw_multi_tensors([t])
        for k in range(2):
            _lib.forge_adamw_advance(sc, step, lr, 0.9, beta2)
            _lib.forge_adamw_multi_step(lst, bits, False, hp, sc)
            torch.cuda.synchronize()
            if bits == 8:
                assert not bool(t["v"].any()) and not bool(t["v_scale"].any())
                assert bool((t["m"] != 0).all()) and bool((t["m_scale"] > 0).all())
            t["grad"].zero_()
        runs[bits] = t["master"].double().cpu().numpy()
    assert np.isfinite(runs[8]).all()
    second = 0.474 * 2.0 ** -7
    bound = lr * (second * (0.71 * 2.0 ** -7 + 255 / 2 / 127.0 ** 2) + 2 * 2.0 ** -7 * 2.0 ** -20)
    # (the new masters, below 2^-6, are rounded to 2^-24 of themselves, twice)
    assert np.max(np.abs(runs[8] - runs[32])) <= bound + 2 * 2.0 ** -30


@pytest.mark.parametrize("seed", [None, 77])
def test_a_small_v_beside_a_huge_one_keeps_a_code(seed):
    """Shares of the block's largest v below what fp32 holds: the lowest code, not none; the
    oracle's codes."""
    import torch
    banner(f"adamw multi huge v seed={seed}")
    t = Tensors([700], 8, False, 8)
    d, h = t.dev[0], t.host[0]
    for name in ("m", "v", "m_scale", "v_scale"):
        d[name].zero_()
        h[name][:] = 0
    g = np.float32(2.0) ** np.random.default_rng(1).integers(-60, -20, 700).astype(np.float32)
    g[5::64] = 2.0 ** 61
    g[9::10] = 0.0
    h["grad"] = g
    d["grad"].copy_(torch.from_numpy(g))
    t.call(None if seed is None else torch.tensor([seed], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    m, v = packed.moments_step(g, h["m"], h["m_scale"], h["v"], h["v_scale"], B1, B2, 0.7)
    um, uv = packed.moment_draws(700, 0, seed)
    for name, (q, s) in dict(m=packed.encode_m(m, um), v=packed.encode_v(v, uv)).items():
        assert np.array_equal(t.got(0, name), q) and np.array_equal(t.got(0, name + "_scale"), s), name
    assert np.array_equal(t.got(0, "v") > 0, v > 0) and (v > 0).sum() > 500
    t.check_guards()
