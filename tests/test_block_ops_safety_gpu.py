"""The block operators' behaviour at their borders on the GPU: a wait that runs out is reported and the next call
works, and no call writes outside the buffers it is given."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
PAD = 8192                                  # guard bytes on each side; keeps 256-byte alignment
RAW = {1: (torch.uint8, 0xA5), 2: (torch.int16, 0x5A5A), 4: (torch.int32, 0x5A5A5A5A)}


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


class Guarded:
    """A tensor inside a patterned buffer; `shift` bytes past the 256-byte alignment."""

    def __init__(self, shape, dtype, shift=0):
        es = torch.empty((), dtype=dtype).element_size()
        raw, self.pat = RAW[es]
        self.n, self.p = int(np.prod(shape)), (PAD + shift) // es
        self.buf = torch.full((self.n + 2 * self.p,), self.pat, dtype=raw, device="cuda")
        self.t = self.buf[self.p:self.p + self.n].view(dtype).view(shape)

    def intact(self):
        return bool((self.buf[:self.p] == self.pat).all()) and bool((self.buf[self.p + self.n:] == self.pat).all())


def guards():
    made = []

    def make(shape, dtype, shift=0):
        made.append(Guarded(shape, dtype, shift))
        return made[-1].t
    return made, make


def rand(shape, dt, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()


def codes(rl, dt):
    return rl.ROLA_BF16 if dt == torch.bfloat16 else rl.ROLA_FP32


# outputs on a 256-byte boundary, and 16 bytes past one (the least the C interface asks for)
@pytest.mark.parametrize("shift", [0, 16])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,d,f", [(1, 24, 40), (5, 1544, 264), (97, 136, 264), (333, 200, 328), (333, 208, 336)])
def test_ffn_writes_inside_its_buffers(rl, m, d, f, dt, shift):
    made, make = guards()
    c = rl.make_ffn_config(m, d, f, dtype=codes(rl, dt))
    ws = make((rl.ffn_workspace(c).numel(),), torch.uint8)
    bws = make((rl.ffn_backward_workspace(c).numel(),), torch.uint8)
    X, Wg, Wu, Wd, dY = rand((m, d), dt), rand((f, d), dt), rand((f, d), dt), rand((d, f), dt), rand((m, d), dt, 1)
    Y, dX = make((m, d), dt, shift), make((m, d), dt, shift)
    G, U = make((m, f), torch.float32, shift), make((m, f), torch.float32, shift)
    dWg, dWu, dWd = make((f, d), dt, shift), make((f, d), dt, shift), make((d, f), dt, shift)
    rl.ffn(c, X, Wg, Wu, Wd, Y, ws)
    plain = Y.clone()
    rl.ffn_train(c, X, Wg, Wu, Wd, Y, G, U, ws)
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, dY, dX, dWg, dWu, dWd, bws)
    torch.cuda.synchronize()
    assert torch.equal(plain, Y)
    assert all(g.intact() for g in made)
    for t in (Y, G, U, dX, dWg, dWu, dWd):
        assert torch.isfinite(t).all()


@pytest.mark.parametrize("shift", [0, 16])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,H,Hk,Lq,Lk,causal,lens", [
    (2, 2, 1, 3, 5, False, [5, 2]), (1, 2, 2, 130, 300, True, None), (2, 4, 2, 300, 131, True, [131, 70]),
    (1, 4, 1, 1, 6000, False, None), (1, 1, 1, 6000, 70, False, None), (2, 1, 1, 257, 900, False, [900, 0])])
def test_attention_writes_inside_its_buffers(rl, B, H, Hk, Lq, Lk, causal, lens, dt, shift):
    made, make = guards()
    c = rl.make_attention_config(B, H, Hk, Lq, Lk, causal, dtype=codes(rl, dt))
    ws = make((rl.attention_workspace(c).numel(),), torch.uint8)
    bws = make((rl.attention_backward_workspace(c).numel(),), torch.uint8)
    q, k, v, dO = rand((B, H, Lq, 128), dt), rand((B, Hk, Lk, 128), dt, 1), rand((B, Hk, Lk, 128), dt, 2), rand((B, H, Lq, 128), dt, 3)
    kv = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse, dq = make(q.shape, dt, shift), make((B, H, Lq), torch.float32, 4 if shift else 0), make(q.shape, dt, shift)
    dk, dv = make(k.shape, dt, shift), make(k.shape, dt, shift)
    rl.attention(c, q, k, v, kv, o, lse, ws)
    rl.attention_backward(c, q, k, v, kv, o, lse, dO, dq, dk, dv, bws)
    torch.cuda.synchronize()
    assert all(g.intact() for g in made)
    for t in (o, dq, dk, dv):
        assert torch.isfinite(t).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,d", [(3, 7), (33, 64), (9, 777), (130, 1536), (2, 5120), (3, 20488), (2, 70000)])
def test_layer_norm_writes_inside_its_buffers(rl, rows, d, dt):
    for shift in (0, 4):
        made, make = guards()
        x, g, b, dy = rand((rows, d), dt), rand((d,), dt, 1), rand((d,), dt, 2), rand((rows, d), dt, 3)
        y, dx = make((rows, d), dt, shift), make((rows, d), dt, shift)
        mean, rstd = make((rows,), torch.float32, shift), make((rows,), torch.float32, shift)
        dg, db = make((d,), torch.float32, shift), make((d,), torch.float32, shift)
        ws = make((rl.layer_norm_backward_workspace(x).numel(),), torch.uint8)
        rl.layer_norm(x, g, b, 1e-6, y, mean, rstd)
        rl.layer_norm_backward(x, g, mean, rstd, dy, dx, dg, db, ws)
        torch.cuda.synchronize()
        assert all(t.intact() for t in made)
        for t in (y, mean, rstd, dx, dg, db):
            assert torch.isfinite(t).all()


@pytest.mark.parametrize("m", [1, 70, 300])
def test_ffn_timeout_is_reported_and_the_next_call_works(rl, m):
    """The hook makes every CTA leave out its first load, so the waits on it run out."""
    X, Wg, Wu, Wd = rand((m, 256), torch.bfloat16), rand((512, 256), torch.bfloat16), rand((512, 256), torch.bfloat16, 1), rand((256, 512), torch.bfloat16)
    c = rl.make_ffn_config(m, 256, 512)
    ws, bws, Y, dX = rl.ffn_workspace(c), rl.ffn_backward_workspace(c), torch.empty_like(X), torch.empty_like(X)
    G, U = torch.zeros((m, 512), device="cuda"), torch.zeros((m, 512), device="cuda")
    grads = [torch.empty_like(t) for t in (Wg, Wu, Wd)]
    c.wait_limit_ms, c.debug_flags = 20, rl.ROLA_DEBUG_SKIP_FIRST_K_COPY
    rl.ffn(c, X, Wg, Wu, Wd, Y, ws)
    assert rl.get_device_status(ws) == rl.ROLA_ERR_TIMEOUT
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, X, dX, *grads, bws)
    assert rl.get_device_status(bws) == rl.ROLA_ERR_TIMEOUT
    c.debug_flags = 0
    rl.ffn(c, X, Wg, Wu, Wd, Y, ws)
    assert rl.get_device_status(ws) == rl.ROLA_OK
    x, wg, wu, wd = (t.double() for t in (X, Wg, Wu, Wd))
    g = x @ wg.t()
    want = (g * torch.sigmoid(g) * (x @ wu.t())) @ wd.t()
    assert (Y.double() - want).norm() <= 8e-3 * want.norm()      # three roundings to bf16 of at most 2^-8 each


@pytest.mark.parametrize("Lq,Lk", [(300, 500), (1, 5000)])
def test_attention_timeout_is_reported_and_the_next_call_works(rl, Lq, Lk):
    q, k, v = rand((2, 2, Lq, 128), torch.bfloat16), rand((2, 2, Lk, 128), torch.bfloat16, 1), rand((2, 2, Lk, 128), torch.bfloat16, 2)
    c = rl.make_attention_config(2, 2, 2, Lq, Lk)
    ws, bws, o, lse = rl.attention_workspace(c), rl.attention_backward_workspace(c), torch.empty_like(q), torch.zeros((2, 2, Lq), device="cuda")
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    c.wait_limit_ms, c.debug_flags = 20, rl.ROLA_DEBUG_SKIP_FIRST_K_COPY
    rl.attention(c, q, k, v, None, o, lse, ws)
    assert rl.get_device_status(ws) == rl.ROLA_ERR_TIMEOUT
    rl.attention_backward(c, q, k, v, None, q, lse, q, dq, dk, dv, bws)
    assert rl.get_device_status(bws) == rl.ROLA_ERR_TIMEOUT
    c.debug_flags = 0
    rl.attention(c, q, k, v, None, o, lse, ws)
    assert rl.get_device_status(ws) == rl.ROLA_OK
    want = torch.softmax(q.double() @ k.double().transpose(2, 3) / 128 ** 0.5, 3) @ v.double()
    assert (o.double() - want).norm() <= 8e-3 * want.norm()
