"""The block operators' C entry points without a GPU: struct layouts, defaults, sizes, and every refusal that
is decided on the host before a launch."""
import ctypes
import os
import subprocess

import pytest

from conftest import ROOT


@pytest.fixture(scope="module")
def rl():
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def test_struct_layouts_match_the_header(rl, tmp_path):
    src = tmp_path / "layout.c"
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{os.path.join(ROOT, "include", "rola.h")}"', 'int main(void) {']
    want = []
    for name, cls in (("rola_ffn_config_t", rl.RolaFfnConfig), ("rola_attention_config_t", rl.RolaAttentionConfig)):
        for f, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(cls, f).offset)
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout
    assert [int(x) for x in out.split()] == want


def test_defaults_and_sizes(rl):
    lib = rl.library()
    assert lib.rola_ffn_config_init(None) == rl.ROLA_ERR_INVALID_ARG
    assert lib.rola_attention_config_init(None) == rl.ROLA_ERR_INVALID_ARG
    c = rl.make_ffn_config(100, 64, 128)
    assert (c.act, c.dtype) == (rl.ROLA_LOWRANK_ACT_SILU, rl.ROLA_BF16)
    fwd, bwd = lib.rola_ffn_workspace_bytes(ctypes.byref(c)), lib.rola_ffn_backward_workspace_bytes(ctypes.byref(c))
    assert fwd >= 256 + 2 * 100 * 128 and bwd >= 256 + 3 * 2 * 100 * 128 and fwd % 256 == bwd % 256 == 0
    a = rl.make_attention_config(1, 4, 2, 1, 8192)
    assert a.d_h == 128 and a.scale == 0.0
    # one row of 2 heads over 8192 keys is split; a long row axis is not
    rows = 4
    split = lib.rola_attention_workspace_bytes(ctypes.byref(a))
    assert split >= 256 + 2 * rows * 128 * 4
    assert lib.rola_attention_workspace_bytes(ctypes.byref(rl.make_attention_config(1, 40, 40, 8192, 512))) == 256
    assert lib.rola_layer_norm_backward_workspace_bytes(100, 64, rl.ROLA_BF16) >= 2 * 64 * 4


@pytest.mark.parametrize("field,value,code", [
    ("tokens", 0, 1), ("tokens", -1, 1), ("tokens", (1 << 22) + 1, 2), ("d_model", 0, 1), ("d_model", 12, 1),
    ("d_model", 1 << 21, 2), ("d_ff", 4, 1), ("d_ff", 100, 1), ("act", 5, 1), ("act", -1, 1), ("dtype", 2, 1),
    ("wait_limit_ms", -1, 1), ("wait_limit_ms", 60001, 1), ("debug_flags", 2, 1)])
def test_ffn_config_refusals(rl, field, value, code):
    lib, c = rl.library(), rl.make_ffn_config(4, 64, 128)
    setattr(c, field, value)
    p = ctypes.c_void_p(4096)
    assert lib.rola_ffn_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.rola_ffn_backward_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.rola_ffn(ctypes.byref(c), *[p] * 6, 1 << 40, None) == code
    assert lib.rola_ffn_train(ctypes.byref(c), *[p] * 8, 1 << 40, None) == code
    assert lib.rola_ffn_backward(ctypes.byref(c), *[p] * 12, 1 << 40, None) == code


@pytest.mark.parametrize("field,value,code", [
    ("B", 0, 1), ("H", 0, 1), ("H_kv", 0, 1), ("H_kv", 3, 1), ("Lq", 0, 1), ("Lk", 0, 1), ("Lk", -5, 1), ("d_h", 64, 2),
    ("d_h", 0, 1), ("causal", 2, 1), ("scale", -1.0, 1), ("scale", float("nan"), 1), ("scale", float("inf"), 1),
    ("dtype", 7, 1), ("wait_limit_ms", 60001, 1), ("debug_flags", 4, 1), ("B", 65536, 2), ("Lk", (1 << 30) + 1, 2),
    ("Lq", 1 << 30, 2)])
def test_attention_config_refusals(rl, field, value, code):
    lib, c = rl.library(), rl.make_attention_config(2, 4, 2, 8, 16)
    setattr(c, field, value)
    p = ctypes.c_void_p(4096)
    assert lib.rola_attention_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.rola_attention_backward_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.rola_attention(ctypes.byref(c), *[p] * 7, 1 << 40, None) == code
    assert lib.rola_attention_backward(ctypes.byref(c), *[p] * 11, 1 << 40, None) == code


def calls(rl):
    """Every entry point with its pointer arguments at 4096 (aligned, never read: each call below is refused), and
    the places of its nullable ones and of its workspace."""
    lib = rl.library()
    f, a = rl.make_ffn_config(4, 64, 128), rl.make_attention_config(2, 4, 2, 8, 16)
    fp, ap = ctypes.byref(f), ctypes.byref(a)
    return {
        "ffn": (lambda p: lib.rola_ffn(fp, *p, 1 << 40, None), 6, (), 5),
        "ffn_train": (lambda p: lib.rola_ffn_train(fp, *p, 1 << 40, None), 8, (), 7),
        "ffn_backward": (lambda p: lib.rola_ffn_backward(fp, *p, 1 << 40, None), 12, (), 11),
        "attention": (lambda p: lib.rola_attention(ap, *p, 1 << 40, None), 7, (3, 5), 6),
        "attention_backward": (lambda p: lib.rola_attention_backward(ap, *p, 1 << 40, None), 11, (3,), 10),
    }


@pytest.mark.parametrize("name", ["ffn", "ffn_train", "ffn_backward", "attention", "attention_backward"])
def test_null_and_misaligned_pointers(rl, name):
    call, n, nullable, ws = calls(rl)[name]
    for i in range(n):
        for bad in (None, 4096 + 2):
            if bad is None and i in nullable:
                continue
            p = [ctypes.c_void_p(4096)] * n
            p[i] = ctypes.c_void_p(bad)
            assert call(p) == (rl.ROLA_ERR_WORKSPACE if i == ws else rl.ROLA_ERR_INVALID_ARG), (name, i, bad)
    lib = rl.library()
    p = ctypes.c_void_p(4096)
    f, a = rl.make_ffn_config(4, 64, 128), rl.make_attention_config(2, 4, 2, 8, 16)
    assert lib.rola_ffn(ctypes.byref(f), *[p] * 6, 255, None) == rl.ROLA_ERR_WORKSPACE
    assert lib.rola_attention(ctypes.byref(a), *[p] * 7, 255, None) == rl.ROLA_ERR_WORKSPACE


def test_layer_norm_refusals(rl):
    lib, p, inv = rl.library(), ctypes.c_void_p(4096), rl.ROLA_ERR_INVALID_ARG
    odd = ctypes.c_void_p(4097)
    fwd = lambda rows=4, d=64, dt=0, x=p, g=p, b=p, eps=1e-6, y=p, m=p, r=p: lib.rola_layer_norm(rows, d, dt, x, g, b, eps, y, m, r, None)  # noqa: E731
    assert fwd(rows=0) == fwd(d=0) == fwd(dt=3) == fwd(x=None) == fwd(y=None) == fwd(m=None) == fwd(r=None) == inv
    assert fwd(eps=-1.0) == fwd(eps=float("nan")) == fwd(x=odd) == fwd(g=odd) == fwd(y=odd) == fwd(m=odd) == inv
    assert fwd(d=(1 << 20) + 1) == fwd(rows=1 << 40) == rl.ROLA_ERR_UNSUPPORTED
    bwd = lambda x=p, g=p, m=p, r=p, dy=p, dx=p, dg=p, db=p, ws=p, n=1 << 40: lib.rola_layer_norm_backward(4, 64, 0, x, g, m, r, dy, dx, dg, db, ws, n, None)  # noqa: E731
    for name in ("x", "m", "r", "dy", "dx", "dg", "db"):
        assert bwd(**{name: None}) == inv and bwd(**{name: odd}) == inv
    assert bwd(ws=None) == bwd(ws=odd) == bwd(n=16) == rl.ROLA_ERR_WORKSPACE
    assert lib.rola_layer_norm_backward_workspace_bytes(0, 64, 0) == 0
