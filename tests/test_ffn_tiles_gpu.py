"""The feed-forward's tensor-core products in tiles of 128 x 256, forward and backward, at sizes where every CTA takes
several tiles: against 64 bits, inside guarded buffers, and when a wait runs out.

The forward takes these tiles from 76 of them on in the down product at the latest (fewer tokens go in tiles of few), and
a GB300 has 152 SMs: the sizes below have up to 693 tiles in a product, more than 16 row tiles, partial tiles in
every direction, and rows that are and are not multiples of 32 bytes.
"""
import pytest
import torch

import test_block_ops_safety_gpu as safety
import test_ffn_gpu as base

pytestmark = pytest.mark.gpu
rl = base.rl
BF = torch.bfloat16


def tiles(n, of):
    return -(-n // of)


# tokens, d_model, d_ff
SIZES = [(1300, 3592, 2056), (1300, 3600, 2064), (2200, 1288, 2568), (4200, 648, 2568), (9800, 64, 264)]


@pytest.mark.parametrize("m,d,f", SIZES)
def test_against_64_bits(rl, m, d, f):
    assert m > 96 and tiles(m, 128) * tiles(d, 256) >= 76
    X, Wg, Wu, Wd, dY = base.inputs_of(m, d, f, BF, seed=m)
    base.check("silu", X, Wg, Wu, Wd, base.run(rl, "silu", X, Wg, Wu, Wd, dY), dY)


@pytest.mark.parametrize("act", ["identity", "tanh", "relu", "gelu"])
def test_feature_maps(rl, act):
    X, Wg, Wu, Wd, dY = base.inputs_of(2200, 1288, 520, BF, seed=1)
    base.check(act, X, Wg, Wu, Wd, base.run(rl, act, X, Wg, Wu, Wd, dY), dY)


def test_same_bits(rl):
    X, Wg, Wu, Wd, dY = base.inputs_of(4200, 648, 2568, BF, seed=2)
    want = base.run(rl, "silu", X, Wg, Wu, Wd, dY)
    for _ in range(10):
        assert all(torch.equal(s, t) for s, t in zip(base.run(rl, "silu", X, Wg, Wu, Wd, dY), want))


@pytest.mark.parametrize("shift", [0, 16])
@pytest.mark.parametrize("m,d,f", [(1300, 1800, 328), (2200, 1296, 1296)])
def test_writes_inside_its_buffers(rl, m, d, f, shift):
    made, make = safety.guards()
    c = rl.make_ffn_config(m, d, f)
    ws, bws = make((rl.ffn_workspace(c).numel(),), torch.uint8), make((rl.ffn_backward_workspace(c).numel(),), torch.uint8)
    X, Wg, Wu, Wd, dY = base.inputs_of(m, d, f, BF, seed=3)
    Y, dX = make((m, d), BF, shift), make((m, d), BF, shift)
    G, U = make((m, f), torch.float32, shift), make((m, f), torch.float32, shift)
    dWg, dWu, dWd = make((f, d), BF, shift), make((f, d), BF, shift), make((d, f), BF, shift)
    rl.ffn_train(c, X, Wg, Wu, Wd, Y, G, U, ws)
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, dY, dX, dWg, dWu, dWd, bws)
    torch.cuda.synchronize()
    assert all(g.intact() for g in made)
    base.check("silu", X, Wg, Wu, Wd, (Y, G, U, dX, dWg, dWu, dWd), dY)


def test_timeout_is_reported_and_the_next_call_works(rl):
    X, Wg, Wu, Wd, dY = base.inputs_of(2200, 1288, 2568, BF, seed=4)
    want = base.run(rl, "silu", X, Wg, Wu, Wd, dY)
    c = rl.make_ffn_config(2200, 1288, 2568)
    c.wait_limit_ms, c.debug_flags = 20, rl.ROLA_DEBUG_SKIP_FIRST_K_COPY
    ws, bws, Y, dX = rl.ffn_workspace(c), rl.ffn_backward_workspace(c), torch.empty_like(X), torch.empty_like(X)
    G, U = (torch.zeros((2200, 2568), device="cuda") for _ in range(2))
    rl.ffn_train(c, X, Wg, Wu, Wd, Y, G, U, ws)
    assert rl.get_device_status(ws) == rl.ROLA_ERR_TIMEOUT
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, dY, dX, *(torch.empty_like(t) for t in (Wg, Wu, Wd)), bws)
    assert rl.get_device_status(bws) == rl.ROLA_ERR_TIMEOUT
    assert all(torch.equal(s, t) for s, t in zip(base.run(rl, "silu", X, Wg, Wu, Wd, dY), want))
