"""A NaN gate shows in the feed-forward's output and gradients, whatever the feature map and the form of the products."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


# few tokens, tiles of few tokens side by side, tiles of 128 x 256 (76 of them), fp32 with few and many tokens
@pytest.mark.parametrize("m,dt", [(3, torch.bfloat16), (200, torch.bfloat16), (9800, torch.bfloat16), (5, torch.float32), (200, torch.float32)])
@pytest.mark.parametrize("act", ["silu", "identity", "tanh", "relu", "gelu"])
def test_a_nan_gate(rl, m, dt, act):
    def rand(*shape, seed=0):
        return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dt).cuda()
    X, Wg, Wu, Wd, dY = rand(m, 64), rand(128, 64, seed=1), rand(128, 64, seed=2), rand(64, 128, seed=3), rand(m, 64, seed=4)
    Wg[77] = float("nan")                            # the gate of one feature; its up projection is finite
    c = rl.make_ffn_config(m, 64, 128, act, rl.ROLA_BF16 if dt == torch.bfloat16 else rl.ROLA_FP32)
    Y, (G, U) = torch.empty_like(X), (torch.empty((m, 128), device="cuda") for _ in range(2))
    ws, bws = rl.ffn_workspace(c), rl.ffn_backward_workspace(c)
    dX, dWg, dWu, dWd = (torch.empty_like(t) for t in (X, Wg, Wu, Wd))
    rl.ffn_train(c, X, Wg, Wu, Wd, Y, G, U, ws)
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, dY, dX, dWg, dWu, dWd, bws)
    assert rl.get_device_status(ws) == rl.ROLA_OK and rl.get_device_status(bws) == rl.ROLA_OK
    assert torch.isnan(G[:, 77]).all() and torch.isfinite(U).all()
    assert torch.isnan(Y).all() and torch.isnan(dX).all()
    here = torch.arange(128, device="cuda") == 77
    for name, t in (("dW_gate", dWg), ("dW_up", dWu), ("dW_down", dWd.t())):
        # phi' of the identity does not depend on the gate
        assert torch.isnan(t[here]).all() or (name, act) == ("dW_gate", "identity"), name
        assert torch.isfinite(t[~here]).all(), name
