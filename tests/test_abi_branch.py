"""CPU checks of the C ABI of LayerNorm, rotary axes and window attention: struct
layouts, size queries, and bad arguments rejected before anything is launched."""
import ctypes
import shutil
import subprocess

import pytest

from paper_2609_13645_amd import _lib

INVALID, UNSUPPORTED, ALIGNMENT = (_lib.FORGE_ERR_INVALID_ARG, _lib.FORGE_ERR_UNSUPPORTED,
                                   _lib.FORGE_ERR_ALIGNMENT)


def status(fn, *args):
    try:
        fn(*args)
    except _lib.ForgeError as e:
        return e.status
    return _lib.FORGE_OK


def test_structs_match_the_c_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"forge_rope_axes_cfg": _lib.RopeAxesCfg,
               "forge_attn_window_cfg": _lib.AttnWindowCfg}
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{_lib.HEADER_PATH}"',
             "int main(void) {", '  printf("%d\\n", FORGE_ROPE_MAX_AXES);']
    for c, py in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({c}));')
        lines += [f'  printf("%zu\\n", offsetof({c}, {f}));' for f, _ in py._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([cc, "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True,
                                          text=True).stdout.split()]
    want = [_lib.ROPE_MAX_AXES]
    for py in structs.values():
        want += [ctypes.sizeof(py)] + [getattr(py, f).offset for f, _ in py._fields_]
    assert got == want


# ------------------------------------------------------------- LayerNorm ----

X, G, B, Y, M, R = (0x100000 * i for i in range(1, 7))


@pytest.mark.parametrize("args,want", [
    ((X, G, B, Y, M, R, 4, 12, 1e-5, 0), INVALID),            # hidden % 8
    ((X, G, B, Y, M, R, 4, 8200, 1e-5, 0), INVALID),
    ((X, G, B, Y, M, R, -1, 16, 1e-5, 0), INVALID),
    ((X, G, B, Y, M, R, 4, 16, -1e-5, 0), INVALID),
    ((X, G, B, Y, M, R, 4, 16, float("nan"), 0), INVALID),
    ((None, G, B, Y, M, R, 4, 16, 1e-5, 0), INVALID),
    ((X, G, B, Y, None, R, 4, 16, 1e-5, 0), INVALID),
    ((X, G, B, Y, M, None, 4, 16, 1e-5, 0), INVALID),
    ((X, G, B, X, M, R, 4, 16, 1e-5, 0), INVALID),            # y is x
    ((X, G, B, X + 16, M, R, 4, 16, 1e-5, 0), INVALID),       # y inside x
    ((X, G, B + 8, Y, M, R, 4, 16, 1e-5, 0), ALIGNMENT),
    ((X + 2, G, B, Y, M, R, 4, 16, 1e-5, 0), ALIGNMENT),
    ((None,) * 6 + (0, 16, 1e-5, 0), _lib.FORGE_OK),          # no rows: no launch
])
def test_layernorm_fwd_refusals(args, want):
    assert status(_lib.forge_layernorm_fwd, *args) == want


def test_layernorm_bwd_refusals():
    ok = dict(x=X, g=G, mean=M, rstd=R, dy=B, resid=None, dx=Y, dg=0x800000, db=0x900000, acc=1,
              tokens=4, hidden=16, ws=0xA00000, stream=0)

    def st(**kw):
        return status(_lib.forge_layernorm_bwd, *dict(ok, **kw).values())
    for name in ("x", "g", "mean", "rstd", "dy", "dx", "dg", "ws"):
        assert st(**{name: None}) == INVALID, name
        assert st(**{name: ok[name] + 8}) == ALIGNMENT, name
    assert st(db=0x900004) == ALIGNMENT and st(resid=0xB00004) == ALIGNMENT
    assert st(dx=X) == INVALID and st(dx=B) == INVALID          # dx over x, over dy
    assert st(resid=Y, dx=Y) == INVALID                         # dx over resid
    assert st(db=0x800000) == INVALID and st(db=0x800020) == INVALID   # db over dg
    assert st(hidden=20) == INVALID and st(tokens=-1) == INVALID
    assert st(tokens=0, x=None, mean=None, rstd=None, dy=None, dx=None, ws=None) == _lib.FORGE_OK
    assert st(tokens=0, dg=None) == INVALID
    with pytest.raises(_lib.ForgeError):
        _lib.forge_layernorm_bwd_workspace_bytes(4, 12)
    assert _lib.forge_layernorm_bwd_workspace_bytes(0, 64) >= 0
    assert 0 < _lib.forge_layernorm_bwd_workspace_bytes(1 << 20, 8192) <= 64 << 20
    assert _lib.forge_layernorm_bwd_workspace_bytes((1 << 31) - 1, 8) > 0


# ----------------------------------------------------------- rotary axes ----

def cfg(d=64, pairs=(8, 12, 12), **kw):
    return _lib.rope_axes_cfg(dict(head_dim=d, pairs=list(pairs), **kw))


@pytest.mark.parametrize("c", [
    dict(pairs=(8, 12, 11)), dict(pairs=(8, 12, 13)), dict(pairs=()), dict(pairs=(32, 0)),
    dict(pairs=(40, -8)), dict(d=24, pairs=(12,)), dict(d=0, pairs=(1,)),
    dict(d=528, pairs=(264,)), dict(d=-64, pairs=(32,))])
def test_rope_axes_cfg_refusals(c):
    assert status(_lib.forge_rope_axes_table, cfg(**c), 16, 1e4, X, Y, 0) == INVALID
    assert status(_lib.forge_rope_axes_apply, cfg(**c), X, 256, Y, 256, G, B, M, 4, 16, 2, 0,
                  0) == INVALID


def test_rope_axes_cfg_bounds():
    with pytest.raises(ValueError):
        _lib.rope_axes_cfg(dict(head_dim=64, pairs=[8, 8, 8, 4, 4]))
    over = cfg()
    over.n_axes = 5
    assert status(_lib.forge_rope_axes_table, over, 16, 1e4, X, Y, 0) == INVALID
    over.n_axes = -1
    assert status(_lib.forge_rope_axes_table, over, 16, 1e4, X, Y, 0) == INVALID
    huge = cfg()
    huge.pairs[0], huge.pairs[1] = (1 << 31) - 1, (1 << 31) - 1   # the sum wraps in 32 bits
    assert status(_lib.forge_rope_axes_table, huge, 16, 1e4, X, Y, 0) == INVALID


def test_rope_axes_table_refusals():
    t = _lib.forge_rope_axes_table
    assert status(t, cfg(), 0, 1e4, X, Y, 0) == INVALID
    assert status(t, cfg(), 16, 0.0, X, Y, 0) == INVALID
    assert status(t, cfg(), 16, float("inf"), X, Y, 0) == INVALID
    assert status(t, cfg(), 16, 1e4, None, Y, 0) == INVALID
    assert status(t, cfg(), 16, 1e4, X, Y + 4, 0) == ALIGNMENT
    assert status(t, cfg(), 1 << 26, 1e4, X, Y, 0) == UNSUPPORTED


def test_rope_axes_apply_refusals():
    ok = dict(x=X, ldx=256, y=Y, ldy=128, cos=G, sin=B, pos=M, tokens=4, n_positions=16, n_rot=2,
              inverse=0, stream=0)

    def st(c=None, **kw):
        return status(_lib.forge_rope_axes_apply, c or cfg(), *dict(ok, **kw).values())
    for name in ("x", "y", "cos", "sin", "pos"):
        assert st(**{name: None}) == INVALID, name
    for name in ("x", "y", "cos", "sin"):
        assert st(**{name: ok[name] + 8}) == ALIGNMENT, name
    assert st(pos=M + 2) == ALIGNMENT
    assert st(ldx=124) == INVALID and st(ldy=132) == INVALID     # below the heads, % 8
    assert st(ldx=120) == INVALID and st(ldy=64) == INVALID
    assert st(n_rot=-1) == INVALID and st(tokens=-1) == INVALID and st(n_positions=0) == INVALID
    assert st(y=X, ldy=128) == INVALID                           # in place, another stride
    assert st(y=X + 256, ldy=256) == INVALID                     # overlapping rows
    assert st(tokens=1 << 30, n_rot=2) == UNSUPPORTED
    assert st(tokens=0, x=None, y=None, pos=None) == _lib.FORGE_OK
    assert st(n_rot=0) == _lib.FORGE_OK


# ------------------------------------------------------- window attention ----

def acfg(**kw):
    return _lib.attn_window_cfg(dict(dict(batch=1, seq=256, n_heads=4, n_kv_heads=2, head_dim=64,
                                          window=64, sinks=4), **kw))


@pytest.mark.parametrize("kw,want", [
    (dict(window=0), INVALID), (dict(window=-5), INVALID), (dict(sinks=-1), INVALID),
    (dict(seq=0), INVALID), (dict(batch=0), INVALID), (dict(n_heads=3), INVALID),
    (dict(n_kv_heads=0), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(seq=(1 << 23) + 1), UNSUPPORTED), (dict(batch=1 << 20, seq=1 << 10), UNSUPPORTED),
    (dict(batch=(1 << 31) - 1, seq=1 << 23), UNSUPPORTED),
    (dict(n_heads=1 << 16, n_kv_heads=1 << 16, seq=1), UNSUPPORTED),
    (dict(batch=1 << 21, seq=1), UNSUPPORTED)])
def test_window_cfg_refusals(kw, want):
    assert status(_lib.forge_attention_window_bwd_workspace_bytes, acfg(**kw)) == want
    assert status(_lib.forge_attention_window_fwd, acfg(**kw), X, None, Y, M, 0) == want
    assert status(_lib.forge_attention_window_bwd, acfg(**kw), X, None, Y, M, G, B, R, 0) == want


def test_window_pointer_refusals():
    f = _lib.forge_attention_window_fwd
    assert status(f, acfg(), None, None, Y, M, 0) == INVALID
    assert status(f, acfg(), X, None, None, M, 0) == INVALID
    assert status(f, acfg(), X, None, Y, None, 0) == INVALID
    assert status(f, acfg(), X, G + 2, Y, M, 0) == ALIGNMENT
    assert status(f, acfg(), X, None, X + 1024, M, 0) == INVALID         # o inside qkv
    b = _lib.forge_attention_window_bwd
    ok = dict(qkv=0x1000000, lens=None, o=0x2000000, lse=0x3000000, do=0x4000000, dqkv=0x5000000,
              ws=0x6000000, stream=0)

    def st(**kw):
        return status(b, acfg(), *dict(ok, **kw).values())
    for name in ("qkv", "o", "lse", "do", "dqkv", "ws"):
        assert st(**{name: None}) == INVALID, name
        assert st(**{name: ok[name] + 8}) == ALIGNMENT, name
    assert st(lens=0x7000001) == ALIGNMENT
    for name in ("qkv", "o", "do"):
        assert st(dqkv=ok[name]) == INVALID, name


def test_window_workspace_is_a_band():
    """The scratch grows with seq x window, not with seq x seq."""
    full = _lib.forge_attention_bwd_workspace_bytes(_lib.AttnCfg(1, 16384, 32, 8, 128))
    w = _lib.forge_attention_window_bwd_workspace_bytes(
        _lib.AttnWindowCfg(1, 16384, 32, 8, 128, 1024, 4))
    assert w < full / 5
    # beyond seq: as seq
    same = [_lib.forge_attention_window_bwd_workspace_bytes(acfg(window=n, sinks=s))
            for n, s in ((256, 256), ((1 << 31) - 1, (1 << 31) - 1))]
    assert same[0] == same[1]


@pytest.mark.parametrize("seq,heads,window,sinks,blocks", [
    # 4 KB blocks of 64 keys x 32 queries of each head: all that a causal tile has
    (16384, 32, 16384, 0, 256 * 512 - 256 * 255), (16384, 32, 1, 16384, 256 * 512 - 256 * 255),
    (16384, 32, 16384, 16384, 256 * 512 - 256 * 255), (3000, 20, 3000, 2, 47 * 94 - 47 * 46),
    # a band that the sequence's end cuts, and the rest of the sinks' rows
    (16384, 32, 8192, 16, 512 + sum(min(258, 512 - 2 * t) for t in range(1, 256))),
    (2050, 64, 1500, 2, 65 + sum(min(49, 65 - 2 * t) for t in range(1, 33))),
    (4128, 16, 100, 130, 129 + 127 + 125 + sum(min(6, 129 - 2 * t) for t in range(3, 65)))])
def test_window_workspace_holds_the_stored_score_gradient_alone(seq, heads, window, sinks, blocks):
    """... beside the statistics, 8 bytes a query and head, and partial sums of up to 192 MB."""
    need = heads * (4096 * blocks + 8 * seq)
    got = _lib.forge_attention_window_bwd_workspace_bytes(
        _lib.AttnWindowCfg(1, seq, heads, heads // 4, 64, window, sinks))
    whole = _lib.forge_attention_bwd_workspace_bytes(_lib.AttnCfg(1, seq, heads, heads // 4, 64))
    assert need <= got <= need + (192 << 20)
    if window >= seq:
        # no sinks before any window, so no sums of theirs
        assert got <= whole + (192 << 20)
        assert seq < 16384 or got <= whole
