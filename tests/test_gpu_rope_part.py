"""GPU parity of forge_rope_part_table / forge_rope_part_apply with the fp64 oracle,
element by element: a rotated value is a sum of two fp32 products of fp32 cos and
sin (below 2^-22 of amplitude (|x1| + |x2|)), rounded once to bf16 (2^-8 of its
value); a passed one keeps its bits."""
import numpy as np
import pytest

import forge_inputs as fi
from oracle import packed
from gpu_util import dev_bf16, host_f64, banner

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
CASES = [
    # tokens, heads, head_dim, rot, offset, interleaved, positions
    (1, 1, 8, 2, 6, False, 4),
    (1, 40, 128, 64, 0, True, 8192),
    (5, 3, 48, 20, 28, False, 300),
    (5, 3, 48, 20, 28, True, 300),
    (333, 5, 64, 64, 0, False, 1000),
    (333, 5, 64, 64, 0, True, 1000),
    (129, 7, 128, 64, 64, False, 64),
    (130, 9, 128, 32, 8, True, 128),
    (77, 4, 128, 48, 16, False, 99),
    (77, 4, 80, 72, 4, True, 99),
    (64, 3, 256, 40, 4, False, 70),
    (19, 2, 512, 512, 0, True, 50),
    (40, 7, 80, 66, 10, False, 90),
    (40, 7, 80, 66, 10, True, 90),
    (4000, 2, 64, 32, 0, False, 5000),
    (1025, 24, 128, 128, 0, False, 2048),
]
SCALINGS = [
    dict(),
    dict(scaling="linear", factor=4.0),
    dict(scaling="base", factor=8.0),
    dict(scaling="parts", factor=8.0, low_turns=1.0, high_turns=32.0, original_positions=4096,
         amplitude=1.25),
]


def _cfg(d, rot, offset=0, inter=False, **kw):
    from paper_2609_13645_amd import _lib
    return _lib.rope_part_cfg(dict(head_dim=d, rot_dim=rot, rot_offset=offset, interleaved=inter,
                                   **kw))


def _tables(c, n, base, factors=None):
    import torch
    from paper_2609_13645_amd import _lib
    cos, sin = (torch.full((n, c.rot_dim // 2), float("nan"), device="cuda") for _ in range(2))
    _lib.forge_rope_part_table(c, factors, n, base, cos, sin)
    return cos, sin


def _frequencies(rot, base, factors=None, **kw):
    names = dict(low_turns="low", high_turns="high", original_positions="original")
    kw = {names.get(k, k): v for k, v in kw.items() if k != "amplitude"}
    return packed.part_frequencies(rot, float(np.float32(base)), pair_factors=factors, **kw)


@pytest.mark.parametrize("rot,base,n,factors,scale", [
    (64, 1e4, 70000, None, SCALINGS[0]), (20, 5e5, 300, None, SCALINGS[1]),
    (128, 1e4, 33000, None, SCALINGS[2]), (64, 5e5, 40000, None, SCALINGS[3]),
    (2, 1e4, 9, [4.0], SCALINGS[1]), (8, 100.0, 1, [1.0, 1.5, 2.0, 64.0], SCALINGS[3])])
def test_tables(rot, base, n, factors, scale):
    """Rounded once from angles in 64 bits, at far positions too."""
    banner(f"rope part table rot={rot} n={n} {scale}")
    cos, sin = _tables(_cfg(128, rot, **scale), n, base, factors)
    amp = scale.get("amplitude", 1.0)
    ang = np.arange(n)[:, None] * _frequencies(rot, base, factors, **scale)
    # half a step of fp32 below 1 (below 2 with an amplitude), and the fp64 angle's own error
    tol = (2.0 ** -25 if amp == 1.0 else 2.0 ** -24) * 1.01 + n * 2.0 ** -49
    assert np.max(np.abs(host_f64(cos) - amp * np.cos(ang))) <= tol
    assert np.max(np.abs(host_f64(sin) - amp * np.sin(ang))) <= tol


def _check(got, x64, pos, c, w, backward, what):
    args = (c.rot_dim, c.rot_offset, bool(c.interleaved))
    ref = packed.rope_part(x64, pos, *args, w, c.amplitude, backward)
    a, b = packed.part_columns(*args)
    size = np.zeros_like(ref)
    size[..., a] = size[..., b] = np.abs(x64[..., a]) + np.abs(x64[..., b])
    bound = np.where(size > 0, HALF * np.abs(ref) + 2.0 ** -22 * c.amplitude * size, 0.0)
    off = np.abs(got.reshape(ref.shape) - ref)
    assert np.all(off <= bound), f"{what}: {float(np.max(off / np.maximum(bound, 1e-300))):.2f}"


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("T,n,d,rot,offset,inter,P", CASES)
def test_rotation(T, n, d, rot, offset, inter, P, backward):
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"rope part T={T} heads={n} d={d} rot={rot}+{offset} inter={inter} back={backward}")
    rng = np.random.default_rng(T + n + d + rot)
    scale = SCALINGS[rot // 2 % 4] if rot > 2 else {}
    c = _cfg(d, rot, offset, inter, **scale)
    cos, sin = _tables(c, P, 1e4)
    w = _frequencies(rot, 1e4, **scale)
    xb = fi.to_bf16_bits(rng.standard_normal((T, (n + 1) * d), dtype=np.float32))
    pos = rng.integers(0, P, T).astype(np.int32)
    pd, x = torch.from_numpy(pos).cuda(), dev_bf16(xb)
    x64 = fi.bf16_bits_to_f64(xb)
    heads = x64[:, :n * d].reshape(T, n, d)
    # into another buffer with rows of another length, in place, and with other heads
    # behind the rotated ones left alone
    y = torch.full((T, n * d + 24), 3.0, dtype=torch.bfloat16, device="cuda")
    _lib.forge_rope_part_apply(c, x, (n + 1) * d, y, n * d + 24, cos, sin, pd, T, P, n, backward)
    torch.cuda.synchronize()
    assert torch.equal(x, dev_bf16(xb)) and bool(torch.all(y[:, n * d:] == 3.0))
    _check(host_f64(y)[:, :n * d], heads, pos, c, w, backward, "apart")
    _lib.forge_rope_part_apply(c, x, (n + 1) * d, x, (n + 1) * d, cos, sin, pd, T, P, n, backward)
    torch.cuda.synchronize()
    assert torch.equal(x[:, :n * d], y[:, :n * d])
    assert np.array_equal(host_f64(x)[:, n * d:], x64[:, n * d:])


def test_positions_clamped_and_left_out():
    import torch
    from paper_2609_13645_amd import _lib
    banner("rope part clamped positions, none")
    T, n, d, rot, P = 90, 2, 64, 32, 40
    c = _cfg(d, rot, 32, True)
    cos, sin = _tables(c, P, 1e4)
    w = _frequencies(rot, 1e4)
    rng = np.random.default_rng(4)
    xb = fi.to_bf16_bits(rng.standard_normal((T, n * d), dtype=np.float32))
    x64 = fi.bf16_bits_to_f64(xb).reshape(T, n, d)
    pos = rng.integers(-2 ** 31, 2 ** 31, T).astype(np.int32)
    pos[:6] = [-1, 0, 39, 40, 2 ** 31 - 1, -2 ** 31]
    y = torch.empty((T, n * d), dtype=torch.bfloat16, device="cuda")
    for p, want in ((torch.from_numpy(pos).cuda(), np.clip(pos, 0, P - 1)),
                    (None, np.arange(T) % P)):
        _lib.forge_rope_part_apply(c, dev_bf16(xb), n * d, y, n * d, cos, sin, p, T, P, n)
        torch.cuda.synchronize()
        _check(host_f64(y), x64, want, c, w, False, "positions")


def test_whole_heads_in_halves_are_plain_rope():
    """forge_rope_apply's bits."""
    import torch
    from paper_2609_13645_amd import _lib
    banner("rope part of whole heads")
    T, n, d, P = 200, 6, 128, 256
    cos, sin = (torch.empty((P, d // 2), device="cuda") for _ in range(2))
    _lib.forge_rope_table(P, d, 5e5, cos, sin)
    rng = np.random.default_rng(8)
    x = dev_bf16(fi.to_bf16_bits(rng.standard_normal((T, n * d), dtype=np.float32)))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    for back in (False, True):
        y = torch.empty_like(x)
        _lib.forge_rope_part_apply(_cfg(d, d), x, n * d, y, n * d, cos, sin, pos, T, P, n, back)
        _lib.forge_rope_apply(x, n * d, cos, sin, pos, T, P, n, d, back)
        torch.cuda.synchronize()
        assert torch.equal(x, y)


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (20, False), (20, True)])
def test_what_is_not_finite_stays_in_its_pair(rot, inter):
    import torch
    from paper_2609_13645_amd import _lib
    banner(f"rope part NaN rot={rot} inter={inter}")
    T, n, d, P = 33, 3, 64, 64
    c = _cfg(d, rot, d - rot, inter)
    cos, sin = _tables(c, P, 1e4)
    x = torch.randn((T, n * d), device="cuda").to(torch.bfloat16)
    y, z = torch.empty_like(x), torch.empty_like(x)
    _lib.forge_rope_part_apply(c, x, n * d, y, n * d, cos, sin, None, T, P, n)
    a, b = packed.part_columns(rot, d - rot, inter)
    at = (17, d + int(a[3]))
    x[at] = float("nan")
    x[20, 5 if rot < d else 2 * d + int(b[1])] = float("inf")
    _lib.forge_rope_part_apply(c, x, n * d, z, n * d, cos, sin, None, T, P, n)
    torch.cuda.synchronize()
    changed = np.argwhere((host_f64(y) != host_f64(z)))
    want = {(17, d + int(a[3])), (17, d + int(b[3]))}
    want |= {(20, 5)} if rot < d else {(20, 2 * d + int(a[1])), (20, 2 * d + int(b[1]))}
    assert {tuple(i) for i in changed.tolist()} == want


def test_rope_part_replayed_from_a_graph_on_another_stream():
    import torch
    from paper_2609_13645_amd import _lib
    banner("rope part graph")
    T, n, d, rot, P = 301, 5, 128, 64, 512
    c = _cfg(d, rot, 0, True)
    cos, sin = _tables(c, P, 1e4)
    x = torch.randn((T, n * d), device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, P, (T,), device="cuda", dtype=torch.int32)
    y, want = torch.empty_like(x), torch.empty_like(x)
    args = (n * d, cos, sin, pos, T, P, n)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        _lib.forge_rope_part_table(c, None, P, 1e4, cos, sin)
        _lib.forge_rope_part_apply(c, x, n * d, y, *args)
    for k in range(3):
        x.copy_(x.flip(0))
        pos.copy_(pos.flip(0))
        cos.zero_()
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        _lib.forge_rope_part_apply(c, x, n * d, want, *args, stream=side)
        side.synchronize()
        assert torch.equal(y, want), k
