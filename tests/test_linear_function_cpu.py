"""What the differentiable linear layer refuses before it looks for a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def rl():
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


X, W = torch.zeros(2, 12, 64), torch.zeros(128, 64)


@pytest.mark.parametrize("shape", [(12, 2, 128), (24, 1, 128), (1, 24, 128), (2, 12, 64), (128,), (1, 128), (2, 1, 128), (2, 6, 256), (48, 64)])
def test_residuals_of_another_arrangement_are_refused(rl, shape):
    with pytest.raises(ValueError, match="residual"):
        rl.LinearFunction.apply(X, W, None, torch.zeros(shape), "identity")


@pytest.mark.parametrize("shape", [(2, 12, 128), (24, 128)])
def test_the_output_s_shape_and_its_rows_are_taken(rl, shape):
    """The next thing that is missing is the GPU."""
    with pytest.raises(ValueError, match="X must be a CUDA tensor"):
        rl.LinearFunction.apply(X, W, None, torch.zeros(shape), "identity")
