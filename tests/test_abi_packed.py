"""CPU checks of the C ABI of the operators of packed training: struct layouts, size
queries, and bad arguments rejected before anything is launched."""
import ctypes
import shutil
import subprocess

import pytest

from paper_2609_13645_amd import _lib

INVALID, UNSUPPORTED, ALIGNMENT, OK = (_lib.FORGE_ERR_INVALID_ARG, _lib.FORGE_ERR_UNSUPPORTED,
                                       _lib.FORGE_ERR_ALIGNMENT, _lib.FORGE_OK)
X, Y, C, S, P = (0x1000000 * i for i in range(1, 6))


def status(fn, *args):
    try:
        fn(*args)
    except _lib.ForgeError as e:
        return e.status
    return OK


def layout(tmp_path, structs, macros=()):
    """The C compiler's sizes, offsets and macro values."""
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{_lib.HEADER_PATH}"',
             "int main(void) {"]
    lines += [f'  printf("%d\\n", (int){m});' for m in macros]
    for c, py in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({c}));')
        lines += [f'  printf("%zu\\n", offsetof({c}, {f}));' for f, _ in py._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([cc, "-o", str(exe), str(src)], check=True)
    return [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True,
                                           text=True).stdout.split()]


def ours(structs):
    return [n for py in structs.values()
            for n in [ctypes.sizeof(py)] + [getattr(py, f).offset for f, _ in py._fields_]]


# ----------------------------------------------------------- rotary part ----

def test_rope_part_struct_matches_the_c_header(tmp_path):
    structs = {"forge_rope_part_cfg": _lib.RopePartCfg}
    names = ["none", "linear", "base", "parts"]
    got = layout(tmp_path, structs, [f"FORGE_ROPE_SCALE_{n.upper()}" for n in names])
    assert got == [_lib.ROPE_SCALINGS[n] for n in names] + ours(structs)


def rcfg(**kw):
    return _lib.rope_part_cfg(dict(dict(head_dim=64, rot_dim=32), **kw))


@pytest.mark.parametrize("kw", [
    dict(head_dim=60), dict(head_dim=0), dict(head_dim=-64), dict(head_dim=520), dict(rot_dim=0),
    dict(rot_dim=31), dict(rot_dim=66), dict(rot_dim=-2), dict(rot_offset=34), dict(rot_offset=1),
    dict(rot_offset=-2), dict(rot_offset=2 ** 31 - 2), dict(amplitude=0.0),
    dict(amplitude=float("inf")), dict(amplitude=float("nan")),
    dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=float("nan")),
    dict(scaling="base", factor=2.0, rot_dim=2), dict(scaling="base", factor=-1.0),
    dict(scaling="parts", factor=2.0, low_turns=1.0, high_turns=1.0, original_positions=9),
    dict(scaling="parts", factor=2.0, low_turns=-1.0, high_turns=1.0, original_positions=9),
    dict(scaling="parts", factor=2.0, low_turns=1.0, high_turns=4.0, original_positions=0),
    dict(scaling="parts", factor=2.0, low_turns=1.0, high_turns=float("inf"),
         original_positions=9)])
def test_rope_part_cfg_refusals(kw):
    assert status(_lib.forge_rope_part_table, rcfg(**kw), None, 16, 1e4, X, Y, 0) == INVALID
    assert status(_lib.forge_rope_part_apply, rcfg(**kw), X, 256, Y, 256, C, S, P, 4, 16, 2, 0,
                  0) == INVALID


def test_rope_part_unknown_scaling():
    c = rcfg()
    for c.scaling in (-1, 4):
        assert status(_lib.forge_rope_part_table, c, None, 16, 1e4, X, Y, 0) == INVALID
    with pytest.raises(KeyError):
        rcfg(scaling="twice")


def test_rope_part_table_refusals():
    t = _lib.forge_rope_part_table
    assert status(t, rcfg(), None, 0, 1e4, X, Y, 0) == INVALID
    assert status(t, rcfg(), None, 16, 0.0, X, Y, 0) == INVALID
    assert status(t, rcfg(), None, 16, float("inf"), X, Y, 0) == INVALID
    assert status(t, rcfg(), None, 16, 1e4, None, Y, 0) == INVALID
    assert status(t, rcfg(), None, 16, 1e4, X, Y + 4, 0) == ALIGNMENT
    assert status(t, rcfg(), None, 1 << 27, 1e4, X, Y, 0) == UNSUPPORTED
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert status(t, rcfg(), [1.0] * 15 + [bad], 16, 1e4, X, Y, 0) == INVALID
    with pytest.raises(ValueError):
        t(rcfg(), [1.0] * 15, 16, 1e4, X, Y, 0)


def test_rope_part_apply_refusals():
    ok = dict(x=X, ldx=256, y=Y, ldy=128, cos=C, sin=S, pos=P, tokens=4, n_positions=16, n_rot=2,
              backward=0, stream=0)

    def st(c=None, **kw):
        return status(_lib.forge_rope_part_apply, c or rcfg(), *dict(ok, **kw).values())
    for name in ("x", "y", "cos", "sin"):
        assert st(**{name: None}) == INVALID, name
        assert st(**{name: ok[name] + 8}) == ALIGNMENT, name
    assert st(pos=P + 2) == ALIGNMENT
    assert st(ldx=124) == INVALID and st(ldy=132) == INVALID     # below the heads, % 8
    assert st(ldx=120) == INVALID and st(ldy=64) == INVALID
    assert st(n_rot=-1) == INVALID and st(tokens=-1) == INVALID and st(n_positions=0) == INVALID
    assert st(y=X, ldy=128) == INVALID                           # in place, another stride
    assert st(y=X + 256, ldy=256) == INVALID                     # overlapping rows
    assert st(tokens=1 << 24) == UNSUPPORTED
    assert st(tokens=0, x=None, y=None, pos=None) == OK
    assert st(n_rot=0) == OK


# ------------------------------------------------- AdamW over many tensors ----

def test_adamw_multi_struct_matches_the_c_header(tmp_path):
    structs = {"forge_adamw_multi_tensor": _lib.AdamwMultiTensor}
    assert layout(tmp_path, structs, ["FORGE_ADAMW_BLOCK"]) == [_lib.ADAMW_BLOCK] + ours(structs)


HP = _lib.AdamwHparams(0.9, 0.95, 1e-8, 0.1)
T8 = dict(master=X, param=Y, grad=C, m=S, v=P, m_scale=0x6000000, v_scale=0x7000000, n=100)
SC, SEED = 0x8000000, 0x9000000


def step(tensors, bits=8, hp=HP, sc=SC, seed=SEED):
    return status(_lib.forge_adamw_multi_step, _lib.adamw_multi_tensors(tensors), bits, 0, hp, sc,
                  seed, 0)


def test_adamw_multi_refusals():
    for name in ("master", "param", "grad", "m", "v"):
        for bits in (8, 32):
            assert step([T8, dict(T8, **{name: None})], bits) == INVALID, name
            assert step([T8, dict(T8, **{name: T8[name] + 8})], bits) == ALIGNMENT, name
    for name in ("m_scale", "v_scale"):
        assert step([dict(T8, **{name: None})]) == INVALID, name
        assert step([dict(T8, **{name: T8[name] + 2})]) == ALIGNMENT, name
    for bits in (0, 16, 4, -8):
        assert step([T8], bits) == INVALID
    assert step([dict(T8, n=-1)]) == INVALID and step([dict(T8, n=1 << 40)]) == UNSUPPORTED
    for bad in (float("nan"), float("inf")):
        assert step([dict(T8, lr_scale=bad)]) == INVALID
        assert step([dict(T8, decay_scale=bad)]) == INVALID
    assert step([T8], sc=None) == INVALID and step([T8], sc=SC + 4) == ALIGNMENT
    assert step([T8], seed=SEED + 1) == ALIGNMENT
    assert step([T8], hp=_lib.AdamwHparams(1.0, 0.95, 1e-8, 0.1)) == INVALID
    assert step([T8], hp=_lib.AdamwHparams(0.9, 0.95, -1e-8, 0.1)) == INVALID
    # nothing to do
    empty = dict(master=None, n=0)
    assert step([]) == OK and step([empty, empty], sc=None) == OK
    f = _lib.load().forge_adamw_multi_step
    import ctypes as ct
    assert f(None, 1, 8, 0, ct.byref(HP), SC, None, None) == INVALID
    assert f(None, -1, 8, 0, ct.byref(HP), SC, None, None) == INVALID
    assert f(None, (1 << 20) + 1, 8, 0, ct.byref(HP), SC, None, None) == UNSUPPORTED
    assert f(None, 0, 8, 0, None, SC, None, None) == INVALID


def test_adamw_multi_read_refusals():
    def read(tensors, m, v):
        p = [None if x is None else _lib.pointers(x) for x in (m, v)]
        return status(_lib.forge_adamw_multi_read, _lib.adamw_multi_tensors(tensors), *p, 0, 0)
    assert read([T8], [None], None) == INVALID and read([T8], None, [None]) == INVALID
    assert read([T8], [X + 8], None) == ALIGNMENT
    for name in ("m", "m_scale"):
        assert read([dict(T8, **{name: None})], [X], None) == INVALID
    for name in ("v", "v_scale"):
        assert read([dict(T8, **{name: None})], None, [X]) == INVALID
    assert read([dict(T8, n=-1)], [X], None) == INVALID
    assert read([T8], None, None) == OK and read([dict(n=0, master=None)], [None], [None]) == OK
    with pytest.raises(ValueError):
        read([T8, T8], [X], None)
