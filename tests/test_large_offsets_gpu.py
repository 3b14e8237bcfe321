"""Tensors of more than 2^31 elements: the far end of each output against the plain form on the same slice."""
import math

import pytest
import torch

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


def rand(*shape, dtype=BF):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_()


def close(a, b, tol):
    assert torch.isfinite(a).all()
    assert (a.double() - b.double()).norm() <= tol * b.double().norm()


@pytest.mark.parametrize("dtype,tol", [(BF, 4e-3), (torch.float32, 1e-5)])
def test_layer_norm(rl, dtype, tol):
    rows, d = 270000, 8192
    x, dy = rand(rows, d, dtype=dtype), rand(rows, d, dtype=dtype)
    assert x.numel() > 2 ** 31
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dg, db = (torch.empty(n, device="cuda") for n in (rows, rows, d, d))
    rl.layer_norm(x, None, None, 1e-6, y, mean, rstd)
    rl.layer_norm_backward(x, None, mean, rstd, dy, dx, dg, db, rl.layer_norm_backward_workspace(x))
    end = x[-64:].double().requires_grad_()
    ref = torch.nn.functional.layer_norm(end, (d,), eps=1e-6)
    ref.backward(dy[-64:].double())
    close(y[-64:], ref.detach(), tol)
    close(dx[-64:], end.grad, tol)
    total = torch.zeros(d, device="cuda", dtype=torch.float64)
    for part in dy.split(30000):
        total += part.double().sum(0)
    assert (db.double() - total).abs().max() <= 1e-3 * math.sqrt(rows)


def test_feed_forward(rl):
    m, d, f = 270000, 64, 8192
    X, Wg, Wu, Wd, dY = rand(m, d), rand(f, d) * 0.1, rand(f, d) * 0.1, rand(d, f) * 0.01, rand(m, d)
    c = rl.make_ffn_config(m, d, f)
    G, U = (torch.empty((m, f), device="cuda") for _ in range(2))
    assert G.numel() > 2 ** 31
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    grads = [torch.empty_like(t) for t in (Wg, Wu, Wd)]
    ws, bws = rl.ffn_workspace(c), rl.ffn_backward_workspace(c)
    rl.ffn_train(c, X, Wg, Wu, Wd, Y, G, U, ws)
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, dY, dX, *grads, bws)
    assert rl.get_device_status(ws) == rl.ROLA_OK and rl.get_device_status(bws) == rl.ROLA_OK
    x, wg, wu, wd = (t.double().requires_grad_() for t in (X[-200:], Wg, Wu, Wd))
    g = x @ wg.t()
    y = (torch.nn.functional.silu(g) * (x @ wu.t())) @ wd.t()
    y.backward(dY[-200:].double())
    close(G[-200:], g.detach(), 1e-5)
    close(Y[-200:], y.detach(), 1e-2)
    close(dX[-200:], x.grad, 1e-2)
    assert all(torch.isfinite(t).all() for t in grads)


def test_attention_of_one_token_over_a_long_cache(rl):
    Hk, Lk, n = 4, 4300000, 4299999
    q, k, v = rand(1, 8, 1, 128), rand(1, Hk, Lk, 128), rand(1, Hk, Lk, 128)
    assert k.numel() > 2 ** 31
    k[:, :, :-100000] = 0                            # and the weight at the far end
    k[:, :, -100000:] += q.view(1, Hk, 2, 128).sum(2, keepdim=True) * 0.7
    k[:, :, n:], v[:, :, n:] = float("nan"), float("inf")
    c = rl.make_attention_config(1, 8, Hk, 1, Lk)
    o, lse, ws = torch.empty_like(q), torch.empty((1, 8, 1), device="cuda"), rl.attention_workspace(c)
    rl.attention(c, q, k, v, torch.tensor([n], dtype=torch.int32, device="cuda"), o, lse, ws)
    assert rl.get_device_status(ws) == rl.ROLA_OK
    for h in range(8):
        s = (k[0, h // 2, :n].float() @ q[0, h, 0].float()).double() / math.sqrt(128)
        p = torch.softmax(s, 0)
        close(lse[0, h], torch.logsumexp(s, 0, keepdim=True), 1e-5)
        close(o[0, h, 0], (p.float() @ v[0, h // 2, :n].float()).double(), 2e-2)


def test_attention_of_many_queries(rl):
    Lq, Lk = 17000000, 40
    q, k, v, dO = rand(1, 1, Lq, 128), rand(1, 1, Lk, 128), rand(1, 1, Lk, 128), rand(1, 1, Lq, 128)
    assert q.numel() > 2 ** 31
    c = rl.make_attention_config(1, 1, 1, Lq, Lk)
    o, lse, ws = torch.empty_like(q), torch.empty((1, 1, Lq), device="cuda"), rl.attention_workspace(c)
    rl.attention(c, q, k, v, None, o, lse, ws)
    dq, dk, dv, bws = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), rl.attention_backward_workspace(c)
    rl.attention_backward(c, q, k, v, None, o, lse, dO, dq, dk, dv, bws)
    assert rl.get_device_status(ws) == rl.ROLA_OK and rl.get_device_status(bws) == rl.ROLA_OK
    a = q[0, 0, -300:].double().requires_grad_()
    want = torch.softmax(a @ k[0, 0].double().t() / math.sqrt(128), 1) @ v[0, 0].double()
    want.backward(dO[0, 0, -300:].double())
    close(o[0, 0, -300:], want.detach(), 1e-2)
    close(dq[0, 0, -300:], a.grad, 2e-2)
    total = torch.zeros((Lk, 128), device="cuda", dtype=torch.float32)
    for i in range(0, Lq, 1000000):
        p = torch.softmax(q[0, 0, i:i + 1000000].float() @ k[0, 0].float().t() / math.sqrt(128), 1)
        total += p.t() @ dO[0, 0, i:i + 1000000].float()
    close(dv[0, 0], total, 2e-2)
    assert torch.isfinite(dk).all()
