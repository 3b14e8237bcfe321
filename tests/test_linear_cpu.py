"""The linear layer's C entry points without a GPU: struct layout, defaults, sizes, and refusals decided before a launch."""
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


def test_struct_layout_matches_the_header(rl, tmp_path):
    fields = [f for f, _ in rl.RolaLinearConfig._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "%s"\nint main(void) {' % os.path.join(ROOT, "include", "rola.h")
                   + "".join('printf("%%zu\\n", offsetof(rola_linear_config_t, %s));' % f for f in fields)
                   + 'printf("%zu\\n", sizeof(rola_linear_config_t)); return 0; }')
    subprocess.run(["gcc", "-std=c99", str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout
    cls = rl.RolaLinearConfig
    assert [int(v) for v in out.split()] == [getattr(cls, f).offset for f in fields] + [ctypes.sizeof(cls)]


def test_defaults_and_sizes(rl):
    lib = rl.library()
    assert lib.rola_linear_config_init(None) == rl.ROLA_ERR_INVALID_ARG
    c = rl.make_linear_config(100, 64, 128)
    assert (c.act, c.dtype) == (rl.ROLA_LOWRANK_ACT_IDENTITY, rl.ROLA_BF16)
    identity = lib.rola_linear_backward_workspace_bytes(ctypes.byref(c))
    gelu = lib.rola_linear_backward_workspace_bytes(ctypes.byref(rl.make_linear_config(100, 64, 128, "gelu")))
    assert lib.rola_linear_workspace_bytes(ctypes.byref(c)) >= 256
    assert gelu >= identity + 2 * 100 * 128 and identity >= 256 + 128 * 4 and identity % 256 == gelu % 256 == 0


@pytest.mark.parametrize("field,value,code", [
    ("tokens", 0, 1), ("tokens", -1, 1), ("tokens", (1 << 22) + 1, 2), ("d_in", 0, 1), ("d_in", 12, 1), ("d_in", 1 << 21, 2), ("d_out", 4, 1),
    ("d_out", 100, 1), ("d_out", 1 << 21, 2), ("act", 5, 1), ("act", -1, 1), ("dtype", 2, 1), ("wait_limit_ms", -1, 1),
    ("wait_limit_ms", 60001, 1), ("debug_flags", 2, 1)])
def test_config_refusals(rl, field, value, code):
    lib, c = rl.library(), rl.make_linear_config(4, 64, 128)
    setattr(c, field, value)
    p = ctypes.c_void_p(4096)
    assert lib.rola_linear_workspace_bytes(ctypes.byref(c)) == lib.rola_linear_backward_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.rola_linear(ctypes.byref(c), *[p] * 6, 1 << 40, None) == code
    assert lib.rola_linear_train(ctypes.byref(c), *[p] * 7, 1 << 40, None) == code
    assert lib.rola_linear_backward(ctypes.byref(c), *[p] * 8, 1 << 40, None) == code


@pytest.mark.parametrize("name,n,nullable", [("rola_linear", 6, (2, 3)), ("rola_linear_train", 7, (2, 3)), ("rola_linear_backward", 8, (4, 5, 6))])
def test_null_and_misaligned_pointers(rl, name, n, nullable):
    lib, c = rl.library(), rl.make_linear_config(4, 64, 128, "silu")
    for i in range(n):
        for bad in (None, 4096 + 2):
            if bad is None and i in nullable:
                continue
            p = [ctypes.c_void_p(4096)] * n
            p[i] = ctypes.c_void_p(bad)
            want = rl.ROLA_ERR_WORKSPACE if i == n - 1 else rl.ROLA_ERR_INVALID_ARG
            assert getattr(lib, name)(ctypes.byref(c), *p, 1 << 40, None) == want, (i, bad)
    p = ctypes.c_void_p(4096)
    assert getattr(lib, name)(ctypes.byref(c), *[p] * n, 255, None) == rl.ROLA_ERR_WORKSPACE
    if name == "rola_linear_backward":
        assert lib.rola_linear_backward(ctypes.byref(c), p, p, p, p, None, None, None, p, 1 << 40, None) == rl.ROLA_ERR_INVALID_ARG


def test_outputs_that_start_where_another_tensor_does(rl):
    """Y may be the residual; every other output in the place of an argument would be read after it is written."""
    lib, c = rl.library(), rl.make_linear_config(64, 64, 64, "silu")
    p = [1 << 20 + i for i in range(8)]
    for name, n, outs, may in (("rola_linear", 6, (4,), {(4, 3)}), ("rola_linear_train", 7, (4, 5), {(4, 3)}),
                               ("rola_linear_backward", 8, (4, 5, 6), set())):
        for i in outs:
            for j in range(n):
                if i == j or (i, j) in may or (j, i) in may:
                    continue
                q = [ctypes.c_void_p(p[j if k == i else k]) for k in range(n)]
                assert getattr(lib, name)(ctypes.byref(c), *q, 1 << 40, None) == rl.ROLA_ERR_INVALID_ARG, (name, i, j)
