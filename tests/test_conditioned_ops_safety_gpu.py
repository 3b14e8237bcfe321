"""Linear layers and residual norms at their borders on the GPU: a wait that runs out is reported and the next call works, no
call writes outside the buffers it is given, calls of several threads are independent, and tensors may pass 2^31 elements."""
import pytest
import torch

from test_block_ops_safety_gpu import codes, guards, rand
from test_large_offsets_gpu import close
from test_threads_gpu import together

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    yield rola
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shift", [0, 16])
@pytest.mark.parametrize("dt", [BF, torch.float32])
@pytest.mark.parametrize("act", ["identity", "gelu"])
@pytest.mark.parametrize("m,k,n", [(1, 24, 40), (3, 1544, 264), (5, 1544, 264), (97, 136, 264), (333, 200, 328), (700, 72, 1096), (4000, 264, 136)])
def test_linear_writes_inside_its_buffers(rl, m, k, n, act, dt, shift):
    made, make = guards()
    c = rl.make_linear_config(m, k, n, act, codes(rl, dt))
    ws, bws = (make((w(c).numel(),), torch.uint8) for w in (rl.linear_workspace, rl.linear_backward_workspace))
    X, W, b, R, dY = rand((m, k), dt), rand((n, k), dt, 1), rand((n,), dt, 2), rand((m, n), dt, 3), rand((m, n), dt, 4)
    Y, dX, dW = make((m, n), dt, shift), make((m, k), dt, shift), make((n, k), dt, shift)
    Z, db = make((m, n), torch.float32, shift), make((n,), torch.float32, shift)
    rl.linear(c, X, W, b, R, Y, ws)
    plain = Y.clone()
    rl.linear_train(c, X, W, b, R, Y, Z, ws)
    rl.linear_backward(c, X, W, Z, dY, dX, dW, db, bws)
    torch.cuda.synchronize()
    assert torch.equal(plain, Y)
    assert all(g.intact() for g in made)
    for t in (Y, Z, dX, dW, db):
        assert torch.isfinite(t).all()


@pytest.mark.parametrize("dt", [BF, torch.float32])
@pytest.mark.parametrize("B,n,d", [(1, 3, 7), (3, 11, 64), (2, 9, 777), (5, 26, 1536), (1, 2, 5120), (2, 3, 8200), (1, 3, 20488)])
def test_residual_norm_writes_inside_its_buffers(rl, B, n, d, dt):
    for shift in (0, 4):
        made, make = guards()
        c = rl.make_residual_norm_config(B, n, d, "layer", "rms", dtype=codes(rl, dt))
        x, h, dout, dy = (rand((B, n, d), dt, i) for i in range(4))
        mod, vec = rand((3, B, d), dt, 5), rand((3, d), dt, 6)
        v = dict(gate=mod[0], scale=mod[1], gamma_h=vec[0], gamma=vec[1], beta=vec[2])
        out, y, dx, dh = (make((B, n, d), dt, shift) for _ in range(4))
        stats, ws = make((B, n, 4), torch.float32), make((rl.residual_norm_backward_workspace(c).numel(),), torch.uint8)
        grads = {"d" + k: make(t.shape, torch.float32, shift) for k, t in v.items()} | {"dshift": make((B, d), torch.float32, shift)}
        rl.residual_norm(c, x, h, out, y, **v, shift=mod[2], stats=stats)
        rl.residual_norm_backward(c, x, h, stats, dout, dy, dx, dh, ws, **v, **grads)
        torch.cuda.synchronize()
        assert all(g.intact() for g in made)
        for t in (out, y, stats, dx, dh, *grads.values()):
            assert torch.isfinite(t).all()


@pytest.mark.parametrize("m,n", [(70, 512), (800, 512), (800, 2048)])
def test_linear_timeout_is_reported_and_the_next_call_works(rl, m, n):
    """The hook makes every CTA leave out its first load, so the waits on it run out."""
    X, W, R = rand((m, 256), BF), rand((n, 256), BF, 1), rand((m, n), BF, 2)
    c = rl.make_linear_config(m, 256, n)
    ws, bws, Y, dX, dW = rl.linear_workspace(c), rl.linear_backward_workspace(c), torch.empty_like(R), torch.empty_like(X), torch.empty_like(W)
    c.wait_limit_ms, c.debug_flags = 20, rl.ROLA_DEBUG_SKIP_FIRST_K_COPY
    rl.linear(c, X, W, None, R, Y, ws)
    assert rl.get_device_status(ws) == rl.ROLA_ERR_TIMEOUT
    for grads in ((dX, None), (None, dW), (dX, dW)):
        rl.linear_backward(c, X, W, None, R, *grads, None, bws)
        assert rl.get_device_status(bws) == rl.ROLA_ERR_TIMEOUT
    c.debug_flags = 0
    rl.linear(c, X, W, None, R, Y, ws)
    rl.linear_backward(c, X, W, None, R, dX, dW, None, bws)
    assert rl.get_device_status(ws) == rl.get_device_status(bws) == rl.ROLA_OK
    x, w, r = X.double(), W.double(), R.double()
    for got, want in ((Y, x @ w.t() + r), (dX, r @ w), (dW, r.t() @ x)):
        assert (got.double() - want).norm() <= 4e-3 * want.norm()        # one rounding of at most 2^-8


def test_linear_layers_of_several_threads(rl):
    def maker(m, k, n):
        def make():
            X, W, b, R = rand((m, k), BF, m), rand((n, k), BF, 1), rand((n,), BF, 2), rand((m, n), BF, 3)
            c, Y = rl.make_linear_config(m, k, n, "gelu"), torch.empty_like(R)
            ws = rl.linear_workspace(c)
            return lambda st: rl.linear(c, X, W, b, R, Y, ws, stream=st), Y
        return make
    together([maker(2, 256, 512), maker(96, 256, 512), maker(40, 512, 256), maker(800, 256, 512), maker(900, 1032, 512)], 1000)


def test_residual_norms_of_several_threads(rl):
    def maker(d, train):
        def make():
            c = rl.make_residual_norm_config(2, 300, d, "layer", "rms")
            x, h, dy, gate = rand((2, 300, d), BF, d), rand((2, 300, d), BF, 1), rand((2, 300, d), BF, 2), rand((2, d), BF, 3)
            out, y, dx, dh = (torch.empty_like(x) for _ in range(4))
            stats, ws = torch.empty((2, 300, 4), device="cuda"), rl.residual_norm_backward_workspace(c)
            dgate = torch.empty((2, d), device="cuda")

            def call(st):
                rl.residual_norm(c, x, h, out, y, gate=gate, stats=stats, stream=st)
                if train:
                    rl.residual_norm_backward(c, x, h, stats, None, dy, dx, dh, ws, gate=gate, dgate=dgate, stream=st)
            return call, dgate if train else y
        return make
    together([maker(2048, False), maker(1536, True), maker(5120, True), maker(777, True), maker(8192, False)], 500)


@pytest.mark.parametrize("dtype,tol", [(BF, 4e-3), (torch.float32, 1e-5)])
def test_residual_norm_of_more_than_2_31_elements(rl, dtype, tol):
    B, n, d = 3, 90000, 8192
    make = lambda: torch.empty((B, n, d), device="cuda", dtype=dtype).normal_()  # noqa: E731
    x, h, dy = make(), make(), make()
    assert x.numel() > 2 ** 31
    mod = torch.empty((2, B, d), device="cuda", dtype=dtype).normal_()
    c = rl.make_residual_norm_config(B, n, d, "layer", "none", dtype=codes(rl, dtype))
    out, y = torch.empty_like(x), torch.empty_like(x)
    stats, ws = torch.empty((B, n, 4), device="cuda"), rl.residual_norm_backward_workspace(c)
    dgate, dshift = torch.empty((B, d), device="cuda"), torch.empty((B, d), device="cuda")
    rl.residual_norm(c, x, h, out, y, gate=mod[0], scale=mod[1], stats=stats)
    ends = [t[-1, -64:].clone() for t in (out, y)]
    rl.residual_norm_backward(c, x, h, stats, None, dy, out, y, ws, gate=mod[0], scale=mod[1], dgate=dgate, dshift=dshift)
    a, b = (t[-1, -64:].double().requires_grad_() for t in (x, h))
    u = a + mod[0, -1].double() * b
    ref = torch.nn.functional.layer_norm(u, (d,), eps=1e-6) * (1 + mod[1, -1].double())
    ref.backward(dy[-1, -64:].double())
    for got, want in zip((*ends, out[-1, -64:], y[-1, -64:]), (u.detach(), ref.detach(), a.grad, b.grad)):
        close(got, want, tol)
    total = sum(part.double().sum(0) for part in dy[-1].split(30000))
    assert (dshift[-1].double() - total).abs().max() <= 1e-3 * n ** 0.5 and torch.isfinite(dgate).all()


def test_linear_of_more_than_2_31_elements(rl):
    m, k, n = 270000, 64, 8192
    X, W, b, dY = (torch.empty(s, device="cuda", dtype=BF).normal_() for s in ((m, k), (n, k), (n,), (m, n)))
    W *= 0.1
    c = rl.make_linear_config(m, k, n, "gelu")
    Y, Z, dX, dW = torch.empty_like(dY), torch.empty((m, n), device="cuda"), torch.empty_like(X), torch.empty_like(W)
    assert Z.numel() > 2 ** 31
    ws, bws = rl.linear_workspace(c), rl.linear_backward_workspace(c)
    rl.linear_train(c, X, W, b, dY, Y, Z, ws)
    rl.linear_backward(c, X, W, Z, dY, dX, dW, None, bws)
    assert rl.get_device_status(ws) == rl.ROLA_OK and rl.get_device_status(bws) == rl.ROLA_OK
    x, w = X[-200:].double().requires_grad_(), W.double()
    z = x @ w.t() + b.double()
    y = torch.nn.functional.gelu(z) + dY[-200:].double()
    y.backward(dY[-200:].double())
    close(Z[-200:], z.detach(), 1e-5)
    close(Y[-200:], y.detach(), 4e-3)
    close(dX[-200:], x.grad, 8e-3)               # dZ and dX are rounded once each
    assert torch.isfinite(dW).all()
