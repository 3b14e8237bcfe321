"""The residual norm's C entry points without a GPU: struct layout, defaults, sizes, refusals decided before a launch, and
the split of the rows into parts."""
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
    fields = [f for f, _ in rl.RolaResidualNormConfig._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "%s"\nint main(void) {' % os.path.join(ROOT, "include", "rola.h")
                   + "".join('printf("%%zu\\n", offsetof(rola_residual_norm_config_t, %s));' % f for f in fields)
                   + 'printf("%zu\\n", sizeof(rola_residual_norm_config_t)); return 0; }')
    subprocess.run(["gcc", "-std=c99", str(src), "-o", str(tmp_path / "layout")], check=True)
    out = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout
    cls = rl.RolaResidualNormConfig
    assert [int(v) for v in out.split()] == [getattr(cls, f).offset for f in fields] + [ctypes.sizeof(cls)]


def test_defaults_and_sizes(rl):
    lib = rl.library()
    assert lib.rola_residual_norm_config_init(None) == rl.ROLA_ERR_INVALID_ARG
    c = rl.RolaResidualNormConfig()
    lib.rola_residual_norm_config_init(ctypes.byref(c))
    assert (c.norm, c.branch_norm, c.mod_stride, c.dtype) == (rl.ROLA_NORM_LAYER, rl.ROLA_NORM_NONE, 0, rl.ROLA_BF16)
    assert c.eps == pytest.approx(1e-6)
    assert lib.rola_residual_norm_backward_workspace_bytes(ctypes.byref(c)) == 0
    c = rl.make_residual_norm_config(2, 100, 64, "rms", "layer")
    n = lib.rola_residual_norm_backward_workspace_bytes(ctypes.byref(c))
    assert n >= 3 * 64 * 4 * 2 and n % 256 == 0


@pytest.mark.parametrize("field,value,code", [
    ("groups", 0, 1), ("rows", 0, 1), ("rows", -3, 1), ("d", 0, 1), ("norm", 3, 1), ("norm", -1, 1), ("branch_norm", 3, 1),
    ("mod_stride", 63, 1), ("mod_stride", -1, 1), ("eps", -1.0, 1), ("eps", float("nan"), 1), ("eps", float("inf"), 1), ("dtype", 2, 1),
    ("d", (1 << 20) + 1, 2), ("rows", 1 << 30, 2)])
def test_config_refusals(rl, field, value, code):
    lib, c = rl.library(), rl.make_residual_norm_config(1 << 11, 4, 64)
    setattr(c, field, value)
    p, q = ctypes.c_void_p(4096), ctypes.c_void_p(8192)
    assert lib.rola_residual_norm_backward_workspace_bytes(ctypes.byref(c)) == 0
    assert lib.rola_residual_norm(ctypes.byref(c), p, p, p, None, p, p, p, p, p, q, p, None) == code
    assert lib.rola_residual_norm_backward(ctypes.byref(c), p, p, p, None, p, p, p, p, p, p, p, q, p, None, p, p, p, p, p, 1 << 50, None) == code


FORWARD = ("x", "h", "gate", "gamma_h", "gamma", "beta", "scale", "shift", "out", "y", "stats")
BACKWARD = ("x", "h", "gate", "gamma_h", "gamma", "beta", "scale", "stats", "dout", "dy", "dx", "dh", "dgate", "dgamma_h", "dgamma",
            "dbeta", "dscale", "dshift", "ws")


def call(rl, names, config=(2, 4, 64, "layer", "rms"), ws_bytes=1 << 40, **changed):
    """The call with a pointer of its own for each argument (aligned, never read: each call here is refused)."""
    c = rl.make_residual_norm_config(*config)
    p = {n: 4096 * (i + 1) for i, n in enumerate(names)} | changed
    a = [ctypes.c_void_p(p[n]) for n in names]
    if names is FORWARD:
        return rl.library().rola_residual_norm(ctypes.byref(c), *a, None)
    return rl.library().rola_residual_norm_backward(ctypes.byref(c), *a, ws_bytes, None)


@pytest.mark.parametrize("changed", [
    dict(x=None), dict(h=None), dict(out=None), dict(y=None), dict(x=4097), dict(gamma=4097), dict(gate=4097), dict(y=4097), dict(stats=4104),
    dict(out=4096, y=4096), dict(h=None, out=None), dict(h=None, out=None, gate=None)])
def test_forward_refusals(rl, changed):
    assert call(rl, FORWARD, **changed) == rl.ROLA_ERR_INVALID_ARG


@pytest.mark.parametrize("config,changed", [
    ((2, 4, 64, "none", "rms"), dict()), ((2, 4, 64, "none", "rms"), dict(y=None)), ((2, 4, 64, "none", "rms"), dict(y=None, gamma=None, beta=None, scale=None)),
    ((2, 4, 64, "layer", "none"), dict()), ((2, 4, 64, "none", "none"), dict(h=None, out=None, y=None, gate=None, gamma_h=None))])
def test_forward_refuses_vectors_without_their_norm(rl, config, changed):
    assert call(rl, FORWARD, config, **changed) == rl.ROLA_ERR_INVALID_ARG


@pytest.mark.parametrize("changed", [
    dict(x=None), dict(stats=None), dict(stats=4104), dict(dx=None), dict(dh=None), dict(h=None), dict(dy=None), dict(dout=None, dy=None),
    dict(dx=4097), dict(dh=4096 * 11), dict(gate=None), dict(gamma_h=None), dict(gamma=None), dict(beta=None), dict(scale=None), dict(dgate=4098),
    dict(dgamma=4098), dict(dshift=4098), dict(dbeta=4098), dict(dscale=4098), dict(dgamma_h=4098)])
def test_backward_refusals(rl, changed):
    assert call(rl, BACKWARD, **changed) == rl.ROLA_ERR_INVALID_ARG


def test_workspace_refusals(rl):
    for bad in (dict(ws=None), dict(ws=4096 + 16), dict(ws_bytes=255)):
        assert call(rl, BACKWARD, **bad) == rl.ROLA_ERR_WORKSPACE


def test_parts_and_samples_have_slots_of_their_own(tmp_path):
    """rn_row and rn_part on the host: the parts cover the rows, rn_part is rn_row's inverse, and no slot i + s is used twice."""
    src = tmp_path / "parts.cu"
    src.write_text('''#include <cstdio>
#include <set>
#include "%s"
using namespace rola;
int main() {
    for (long long groups : {1LL, 2LL, 3LL, 7LL, 40LL, 1000LL})
        for (long long rows : {1LL, 2LL, 5LL, 13LL, 997LL})
            for (int parts : {1, 2, 3, 31, 152, 1216, 4864}) {
                const long long total = groups * rows;
                if (parts > total) continue;
                if (rn_row(total, parts, 0) != 0 || rn_row(total, parts, parts) != total) return 1;
                std::set<long long> used;
                for (int i = 0; i < parts; ++i) {
                    const long long r0 = rn_row(total, parts, i), r1 = rn_row(total, parts, i + 1);
                    if (r0 >= r1) return 2;
                    for (long long r = r0; r < r1; ++r)
                        if (rn_part(total, parts, r) != i) return 3;
                    for (long long s = r0 / rows; s <= (r1 - 1) / rows; ++s)
                        if (i + s >= parts + groups - 1 || !used.insert(i + s).second) return 4;
                }
            }
    puts("ok");
}''' % os.path.join(ROOT, "paper_2609_06712_gb300", "csrc", "residual_norm.cuh"))
    from paper_2609_06712_gb300 import build
    subprocess.run([build.nvcc(), "-std=c++17", str(src), "-o", str(tmp_path / "parts")], check=True, capture_output=True)
    assert subprocess.run([str(tmp_path / "parts")], capture_output=True, text=True).stdout.strip() == "ok"
