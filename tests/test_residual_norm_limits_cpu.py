"""The bound of the residual norm's waits and its test hook, as the other block operators have them, without a GPU."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def rl():
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


@pytest.mark.parametrize("field,value,good", [("wait_limit_ms", 0, True), ("wait_limit_ms", 60000, True), ("wait_limit_ms", 60001, False),
                                              ("wait_limit_ms", -1, False), ("debug_flags", 1, True), ("debug_flags", 2, False), ("debug_flags", -1, False)])
def test_config(rl, field, value, good):
    lib, c = rl.library(), rl.make_residual_norm_config(2, 4, 64)
    assert (c.wait_limit_ms, c.debug_flags) == (0, 0)
    setattr(c, field, value)
    assert (lib.rola_residual_norm_backward_workspace_bytes(ctypes.byref(c)) > 0) == good
    if not good:
        p = [ctypes.c_void_p(4096 * (i + 1)) for i in range(19)]
        for i in (4, 5, 6, 7):
            p[i] = None
        assert lib.rola_residual_norm(ctypes.byref(c), *p[:11], None) == rl.ROLA_ERR_INVALID_ARG
        assert lib.rola_residual_norm_backward(ctypes.byref(c), *p, 1 << 40, None) == rl.ROLA_ERR_INVALID_ARG
