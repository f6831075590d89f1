"""GPU parity of forge_layernorm_fwd / forge_layernorm_bwd with the fp64 oracle,
element by element.

An output in bf16 is off by at most half a step, 2^-8 of its value. The fp32
arithmetic before it adds roundings of 2^-24 of each term: of the largest
operands (x - mean), and of sums, whose terms pass at most 128 sequential
additions in a lane and ten more across lanes and waves, below 2^-16 of the sum
of the terms' magnitudes with the roundings of the terms themselves.
"""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import branch
from gpu_util import dev_bf16, host_f64, banner

pytestmark = pytest.mark.gpu

HALF, SUM = 2.0 ** -8, 2.0 ** -16
EPS = 1e-5
SIZES = [(1, 8), (1, 8192), (37, 24), (300, 520), (64, 512), (999, 2056), (130, 1000), (5, 4104),
         (2050, 1024), (700, 4096), (9000, 264), (3, 6160),
         # backward: the most rows of one workgroup, and one more
         (24, 520), (12, 1032), (6, 2056), (3, 8192), (25, 72)]


def _bits(rng, shape, std=1.0, mean=0.0):
    return fi.to_bf16_bits((mean + std * rng.standard_normal(shape)).astype(np.float32))


def _inputs(T, h, seed, offset=1.0):
    rng = np.random.default_rng(seed)
    b = dict(x=fi.to_bf16_bits((rng.standard_normal((T, h)) + offset * rng.standard_normal((T, 1)))
                               .astype(np.float32)),
             g=_bits(rng, h, 0.3, 1.0), b=_bits(rng, h, 0.5), dy=_bits(rng, (T, h), 0.1),
             resid=_bits(rng, (T, h), 0.1))
    return {n: dev_bf16(v) for n, v in b.items()}, {n: fi.bf16_bits_to_f64(v)
                                                    for n, v in b.items()}


def _within(got, ref, bound, what):
    off = np.abs(host_f64(got).reshape(ref.shape) - ref)
    worst = float(np.max(off / bound)) if off.size else 0.0
    assert np.all(off <= bound), f"{what}: {worst:.2f} of its bound"


def _fwd(x, g, b, T, h):
    import torch
    from paper_2609_13645_amd import _lib
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    _lib.forge_layernorm_fwd(x, g, b, y, mean, rstd, T, h, EPS)
    torch.cuda.synchronize()
    return y, mean, rstd


@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("T,h", SIZES)
def test_layernorm_fwd(T, h, bias):
    banner(f"layernorm fwd T={T} h={h} bias={bias}")
    d, r = _inputs(T, h, T * 7 + h)
    y, mean, rstd = _fwd(d["x"], d["g"], d["b"] if bias else None, T, h)
    b = r["b"] if bias else np.zeros(h)
    ref, m, rs = branch.layernorm_fwd(r["x"], r["g"], b, EPS)
    size = np.abs(r["x"]).mean(axis=1)
    _within(mean, m, SUM * size + 1e-30, "mean")
    _within(rstd, rs, SUM * rs, "rstd")
    terms = (np.abs(r["x"]) + np.abs(m)[:, None]) * rs[:, None] * np.abs(r["g"]) + np.abs(b)
    _within(y, ref, HALF * np.abs(ref) + SUM * terms, "y")


def test_layernorm_of_rows_far_from_zero_and_of_equal_values():
    """The variance is that of the centred values: a row at 1000 +- 4 keeps its
    statistics, and rows of one value have y = b."""
    banner("layernorm centred variance")
    T, h = 6, 1024
    rng = np.random.default_rng(9)
    x = 1000.0 + 4.0 * rng.integers(-2, 3, (T, h))
    x[4], x[5] = 0.0, -7.0
    xb = fi.to_bf16_bits(x.astype(np.float32))
    _, r = _inputs(T, h, 1)
    g, b = dev_bf16(fi.to_bf16_bits(np.full(h, 2.0, np.float32))), np.full(h, 0.5)
    y, mean, rstd = _fwd(dev_bf16(xb), g, dev_bf16(fi.to_bf16_bits(b.astype(np.float32))), T, h)
    x64 = fi.bf16_bits_to_f64(xb)
    _, m, rs = branch.layernorm_fwd(x64, np.full(h, 2.0), b, EPS)
    _within(mean, m, SUM * np.abs(x64).mean(axis=1) + 1e-30, "mean")
    # the mean's error enters the variance squared: (1000 2^-16)^2 of about 8
    _within(rstd, rs, rs * (SUM + (1000 * SUM) ** 2 / 8.0), "rstd")
    assert np.all(host_f64(y)[4:] == 0.5)


@pytest.mark.parametrize("bias,resid,acc", [(True, False, False), (True, True, True),
                                            (False, True, False)])
@pytest.mark.parametrize("T,h", SIZES)
def test_layernorm_bwd(T, h, bias, resid, acc):
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"layernorm bwd T={T} h={h} bias={bias} resid={resid} accumulate={acc}")
    d, r = _inputs(T, h, T * 5 + h + 1)
    _, m, rs = branch.layernorm_fwd(r["x"], r["g"], None, EPS)
    m, rs = m.astype(np.float32), rs.astype(np.float32)
    ws = torch.full((_lib.forge_layernorm_bwd_workspace_bytes(T, h) // 4,), float("nan"),
                    device="cuda")
    dx = torch.full_like(d["x"], float("nan"))
    first = 0.25 if acc else float("nan")
    dg, db = (torch.full((h,), first, device="cuda") for _ in range(2))
    _lib.forge_layernorm_bwd(d["x"], d["g"], torch.from_numpy(m).cuda(),
                             torch.from_numpy(rs).cuda(), d["dy"], d["resid"] if resid else None,
                             dx, dg, db if bias else None, acc, T, h, ws)
    torch.cuda.synchronize()
    m, rs = m.astype(np.float64), rs.astype(np.float64)
    ref_x, ref_g, ref_b = branch.layernorm_bwd(r["x"], r["g"], m, rs, r["dy"])
    size = (np.abs(r["x"]) + np.abs(m)[:, None]) * rs[:, None]      # of xh's operands
    u = np.abs(r["dy"] * r["g"])
    terms = rs[:, None] * (u + u.mean(1, keepdims=True)
                           + size * (u * size).mean(1, keepdims=True))
    if resid:
        ref_x, terms = ref_x + r["resid"], terms + np.abs(r["resid"])
    _within(dx, ref_x, HALF * np.abs(ref_x) + SUM * terms, "dx")
    # sums over rows: at most T / 2048 + 64 additions one after another
    start, rows = (0.25 if acc else 0.0), SUM + (T / 2048 + 64) * 2.0 ** -24
    _within(dg, ref_g + start, rows * ((np.abs(r["dy"]) * size).sum(0) + start), "dg")
    if bias:
        _within(db, ref_b + start, rows * (np.abs(r["dy"]).sum(0) + start), "db")
    else:
        assert bool(torch.all(db == 0.25)) if acc else bool(torch.isnan(db).all())


@pytest.mark.parametrize("h", [256, 2056, 8192])
def test_layernorm_bwd_of_rows_of_one_value(h):
    """x equals its mean: xh is 0 exactly, however large rstd, so dg is 0 and dx that of
    the centred u."""
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"layernorm bwd rows of one value h={h}")
    T = 77
    d, r = _inputs(T, h, h)
    value = torch.linspace(-700, 900, T, device="cuda").to(torch.bfloat16)
    x = value[:, None].expand(T, h).contiguous()
    m, rs = value.float(), torch.full((T,), EPS ** -0.5, device="cuda")
    ws = torch.empty(_lib.forge_layernorm_bwd_workspace_bytes(T, h), dtype=torch.uint8,
                     device="cuda")
    dx = torch.full_like(x, float("nan"))
    dg, db = (torch.full((h,), float("nan"), device="cuda") for _ in range(2))
    _lib.forge_layernorm_bwd(x, d["g"], m, rs, d["dy"], None, dx, dg, db, False, T, h, ws)
    torch.cuda.synchronize()
    assert not dg.any()
    u, scale = r["dy"] * r["g"], float(rs[0])
    ref = scale * (u - u.mean(1, keepdims=True))
    terms = scale * (np.abs(u) + np.abs(u).mean(1, keepdims=True))
    _within(dx, ref, HALF * np.abs(ref) + SUM * terms, "dx")


def test_layernorm_bwd_repeats_bit_for_bit_and_without_rows():
    import torch
    from paper_2609_13645_amd import _lib
    banner("layernorm bwd determinism")
    T, h = 3001, 1032
    d, r = _inputs(T, h, 3)
    _, m, rs = branch.layernorm_fwd(r["x"], r["g"], None, EPS)
    m, rs = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (m, rs))
    ws = torch.empty(_lib.forge_layernorm_bwd_workspace_bytes(T, h), dtype=torch.uint8,
                     device="cuda")
    out = []
    for _ in range(3):
        dx, dg, db = torch.empty_like(d["x"]), *(torch.empty(h, device="cuda") for _ in range(2))
        _lib.forge_layernorm_bwd(d["x"], d["g"], m, rs, d["dy"], None, dx, dg, db, False, T, h, ws)
        out.append((dx, dg, db))
    torch.cuda.synchronize()
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))
    dg, db = out[0][1:]
    kept = dg.clone()
    _lib.forge_layernorm_bwd(None, None, None, None, None, None, None, dg, db, True, 0, h, None)
    torch.cuda.synchronize()
    assert torch.equal(dg, kept)
    _lib.forge_layernorm_bwd(None, None, None, None, None, None, None, dg, db, False, 0, h, None)
    torch.cuda.synchronize()
    assert not dg.any() and not db.any()


def test_layernorm_of_more_rows_than_a_launch_holds():
    """2^25 + 3 rows of 8: the forward's workgroups take several turns."""
    import torch
    from paper_2609_13645_amd import _lib
    T, h = (1 << 25) + 3, 8
    banner(f"layernorm fwd T={T} h={h}")
    x = torch.randn((T, h), device="cuda").to(torch.bfloat16)
    g, b = (torch.randn(h, device="cuda").to(torch.bfloat16) for _ in range(2))
    y, mean, rstd = _fwd(x, g, b, T, h)
    for at in (0, (1 << 24) - 100, T - 1000):
        rows = slice(at, at + 1000)
        xr = x[rows].double()
        m = xr.mean(1, keepdim=True)
        rs = ((xr - m).square().mean(1, keepdim=True) + EPS).rsqrt()
        ref = (xr - m) * rs * g.double() + b.double()
        terms = (xr.abs() + m.abs()) * rs * g.double().abs() + b.double().abs()
        off = (y[rows].double() - ref).abs()
        assert bool((off <= HALF * ref.abs() + SUM * terms).all()), at
        assert bool(((rstd[rows].double() - rs[:, 0]).abs() <= SUM * rs[:, 0]).all()), at
    assert bool(torch.isfinite(mean).all()) and bool(torch.isfinite(y).all())
