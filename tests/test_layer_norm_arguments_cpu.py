"""Arguments that the differentiable layer norm refuses before anything is launched."""
import pytest
import torch


def test_one_of_gamma_and_beta_alone_is_refused():
    """The gradient of a lone beta would otherwise be left out without a word."""
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    x, one = torch.zeros(4, 64, requires_grad=True), torch.ones(64, requires_grad=True)
    for gamma, beta in ((one, None), (None, one)):
        with pytest.raises(ValueError, match="both tensors or both None"):
            rola.LayerNormFunction.apply(x, gamma, beta, 1e-6)
