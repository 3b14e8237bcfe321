"""The operators together in a DiT block: its forward pass and gradients against the same block in 64-bit torch (the
RoLA self-attention aside, whose output both use), and a few training steps."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block_mod():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import dit_block
    return dit_block


def test_block_matches_torch_in_64_bits(block_mod, monkeypatch):
    from paper_2609_06712_gb300 import configs, rola
    torch.manual_seed(1)
    cfg = configs.get("tiny", B=2, T=2, Hh=5, Ww=9, keep=1.0)      # every block kept: no decision near a tie
    block = block_mod.DiTBlock(cfg, d_text=96, d_ff=328, dtype=torch.float32)
    x, dy = (torch.randn(2, cfg["N"], 256, device="cuda") for _ in range(2))
    text, n = torch.randn(2, 31, 96, device="cuda"), torch.tensor([31, 7], dtype=torch.int32, device="cuda")
    x.requires_grad_()
    block(x, text, n).backward(dy)
    got = {name: p.grad for name, p in block.named_parameters()} | {"x": x.grad}

    # the same graph in 64 bits; the module under RoLA keeps its own kernels and gradients (fp32)
    class Rola64(torch.autograd.Function):
        @staticmethod
        def forward(ctx, c, *t):
            with torch.enable_grad():
                ctx.leaves = [a.detach().float().requires_grad_() for a in t[:5]]
                ctx.out = real(c, *ctx.leaves, None)
            return ctx.out.detach().double()

        @staticmethod
        def backward(ctx, g):
            return None, *(t.double() for t in torch.autograd.grad(ctx.out, ctx.leaves, g.float())), None
    real = rola.RoLAFunction.apply

    def attention(q, k, v, lens, causal):
        s = q @ k.transpose(2, 3) / math.sqrt(128)
        seen = torch.arange(k.shape[2], device="cuda")[None, :] < lens[:, None]
        return torch.softmax(s.masked_fill(~seen[:, None, None], float("-inf")), 3) @ v

    def ffn(t, g, u, d, act):
        lin = torch.nn.functional.linear
        return lin(torch.nn.functional.silu(lin(t, g)) * lin(t, u), d)
    for name, f in (("RoLAFunction", Rola64.apply), ("AttentionFunction", attention), ("FfnFunction", ffn), (
            "LayerNormFunction", lambda t, g, b, eps: torch.nn.functional.layer_norm(t, t.shape[-1:], g, b, eps))):
        monkeypatch.setattr(rola, name, type("Plain", (), {"apply": staticmethod(f)}))
    ref = block_mod.DiTBlock(cfg, d_text=96, d_ff=328, dtype=torch.float32).double()
    ref.load_state_dict(block.state_dict())
    x64 = x.detach().double().requires_grad_()
    ref(x64, text.double(), n).backward(dy.double())
    want = {name: p.grad for name, p in ref.named_parameters()} | {"x": x64.grad}
    for name in want:
        err = (got[name].double() - want[name]).norm() / want[name].norm()
        # fp32 throughout; torch's fp32 projections and the module's gradients (bar 1e-5 each) lie between
        assert err <= 1e-4, (name, err.item())


def test_training_lowers_the_loss(block_mod):
    losses = block_mod.train(6)
    assert all(math.isfinite(v) for v in losses) and losses[-1] < losses[0]
