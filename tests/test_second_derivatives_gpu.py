"""The differentiable ops have first derivatives only: asking for one of a gradient raises, where a constant in its place
would lose terms of a sum without a word."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import configs, inputs, rola

    def leaf(*shape, seed=0):
        return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda().requires_grad_()
    cfg = configs.get("tiny")
    x = inputs.make_inputs(cfg, dtype=torch.float32)
    x = {n: t.cuda().requires_grad_() for n, t in x.items() if n in ("q", "k", "v", "P_q", "P_k")}
    return {
        "layer_norm": (lambda a, g, b: rola.LayerNormFunction.apply(a, g, b, 1e-6), [leaf(6, 64), leaf(64), leaf(64, seed=1)]),
        "ffn": (lambda *t: rola.FfnFunction.apply(*t, "silu"), [leaf(6, 64), leaf(128, 64), leaf(128, 64, seed=1), leaf(64, 128)]),
        "attention": (lambda *t: rola.AttentionFunction.apply(*t, None, False),
                      [leaf(1, 2, 5, 128), leaf(1, 2, 7, 128), leaf(1, 2, 7, 128, seed=1)]),
        "rola": (lambda *t: rola.RoLAFunction.apply(rola.make_config(cfg, rola.ROLA_FP32), *t, None),
                 [x[n] for n in ("q", "k", "v", "P_q", "P_k")]),
    }


@pytest.mark.parametrize("name", ["layer_norm", "ffn", "attention", "rola"])
def test_a_gradient_of_a_gradient_raises(ops, name):
    f, leaves = ops[name]
    plain = torch.autograd.grad(f(*leaves).square().sum(), leaves)
    grads = torch.autograd.grad(f(*leaves).square().sum(), leaves, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(plain, grads))
    # a penalty on the gradients beside a term that has an ordinary derivative
    total = sum(g.square().sum() for g in grads) + leaves[0].sum()
    with pytest.raises(RuntimeError, match="once_differentiable"):
        total.backward()
