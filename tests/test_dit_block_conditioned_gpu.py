"""The operators together in a conditioned DiT block, its linear layers and gated norms among them: forward pass and
gradients against the same block in 64-bit torch (the RoLA self-attention aside, whose output both use), and training steps."""
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


def plain64(rola):
    """The library's differentiable ops in 64-bit torch, by name; the module keeps its own kernels and gradients (fp32)."""
    fn = torch.nn.functional
    real = rola.RoLAFunction.apply

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

    def attention(q, k, v, lens, causal):
        s = q @ k.transpose(2, 3) / math.sqrt(128)
        seen = torch.arange(k.shape[2], device="cuda")[None, :] < lens[:, None]
        return torch.softmax(s.masked_fill(~seen[:, None, None], float("-inf")), 3) @ v

    def residual_norm(x, h, gate, gamma_h, gamma, beta, scale, shift, norm, branch, eps):
        u = x if h is None else x + (h if gate is None else gate[:, None] * h)
        if norm == "none":
            return u, None
        y = fn.layer_norm(u, u.shape[-1:], gamma, beta, eps)
        return (None if h is None else u), (y if scale is None else y * (1 + scale[:, None]) + shift[:, None])
    return dict(RoLAFunction=Rola64.apply, AttentionFunction=attention, ResidualNormFunction=residual_norm,
                FfnFunction=lambda t, g, u, d, act: fn.linear(fn.silu(fn.linear(t, g)) * fn.linear(t, u), d),
                LinearFunction=lambda t, w, b, r, act: fn.linear(t, w, b))


def test_block_matches_torch_in_64_bits(block_mod, monkeypatch):
    from paper_2609_06712_gb300 import configs, rola
    torch.manual_seed(1)
    cfg = configs.get("tiny", B=2, T=2, Hh=5, Ww=9, keep=1.0)      # every block kept: no decision near a tie
    block = block_mod.DiTBlock(cfg, d_text=96, d_ff=328, dtype=torch.float32, d_cond=72)
    x, dy = (torch.randn(2, cfg["N"], 256, device="cuda") for _ in range(2))
    text, n = torch.randn(2, 31, 96, device="cuda"), torch.tensor([31, 7], dtype=torch.int32, device="cuda")
    cond = torch.randn(2, 72, device="cuda").requires_grad_()
    x.requires_grad_()
    out = block(x, text, n, cond)
    out.backward(dy)
    got = {name: p.grad for name, p in block.named_parameters()} | {"x": x.grad, "cond": cond.grad, "out": out.detach()}
    for name, f in plain64(rola).items():
        monkeypatch.setattr(rola, name, type("Plain", (), {"apply": staticmethod(f)}))
    ref = block_mod.DiTBlock(cfg, d_text=96, d_ff=328, dtype=torch.float32, d_cond=72).double()
    ref.load_state_dict(block.state_dict())
    x64, cond64 = (t.detach().double().requires_grad_() for t in (x, cond))
    out64 = ref(x64, text.double(), n, cond64)
    out64.backward(dy.double())
    want = {name: p.grad for name, p in ref.named_parameters()} | {"x": x64.grad, "cond": cond64.grad, "out": out64.detach()}
    for name in want:
        err = (got[name].double() - want[name]).norm() / want[name].norm()
        # fp32 throughout; the module's gradients (bar 1e-5) lie between
        assert err <= 1e-4, (name, err.item())


def test_block_in_bf16_is_near_the_one_in_fp32(block_mod):
    """The same weights in both types: the tensor-core path through every operator.  Some thirty roundings of at most 2^-8
    relative lie between; taken as independent they come to 30^(1/2) 2^-8 = 2.1 %, and 8 % is four times that."""
    from paper_2609_06712_gb300 import configs
    torch.manual_seed(2)
    cfg = configs.get("tiny", B=2, T=2, Hh=8, Ww=20, keep=1.0)
    fp32 = block_mod.DiTBlock(cfg, d_text=192, d_ff=704, dtype=torch.float32, d_cond=128)
    with torch.no_grad():
        for p in fp32.parameters():
            p.copy_(p.bfloat16())
    bf16 = block_mod.DiTBlock(cfg, d_text=192, d_ff=704, d_cond=128)
    bf16.load_state_dict(fp32.state_dict())
    x, text, cond, dy = (torch.randn(s, device="cuda").bfloat16() for s in ((2, cfg["N"], 256), (2, 77, 192), (2, 128), (2, cfg["N"], 256)))
    results = []
    for block, dt in ((fp32, torch.float32), (bf16, torch.bfloat16)):
        out = block(x.to(dt), text.to(dt), None, cond.to(dt))
        out.backward(dy.to(dt))
        results.append([out.detach()] + [p.grad for p in block.parameters()])
    for a, b in zip(*results):
        assert torch.isfinite(b).all() and (a.double() - b.double()).norm() <= 0.08 * a.double().norm()


@pytest.mark.parametrize("conditioned", [False, True])
def test_training_steps_run(block_mod, conditioned):
    losses = block_mod.train(3, conditioned=conditioned)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)


def test_a_step_captured_into_a_graph(block_mod):
    """Forward and backward of the conditioned block captured and replayed: the gradients of the eager step."""
    from paper_2609_06712_gb300 import configs
    torch.manual_seed(3)
    cfg = configs.get("tiny", T=2, Hh=5, Ww=9, keep=1.0)
    block = block_mod.DiTBlock(cfg, d_text=96, d_ff=328, d_cond=64)
    x, text, cond, dy = (torch.randn(s, device="cuda").bfloat16() for s in ((1, cfg["N"], 256), (1, 31, 96), (1, 64), (1, cfg["N"], 256)))
    params = list(block.parameters())

    def step():
        out = block(x, text, None, cond)
        return [out, *torch.autograd.grad(out, params, dy)]
    want = [t.detach().clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
