"""What a DiT block asks of its conditioning vector, decided before any kernel runs."""
import pytest
import torch


@pytest.mark.parametrize("d_cond,shape", [(64, None), (64, (2, 32)), (64, (1, 64)), (64, (2, 1, 64)), (None, (2, 64))])
def test_a_conditioning_vector_of_another_shape_is_refused(d_cond, shape):
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import configs, dit_block
    cfg = configs.get("tiny")
    block = dit_block.DiTBlock(cfg, d_text=64, d_ff=64, device="cpu", d_cond=d_cond)
    x, text = torch.zeros(2, cfg["N"], cfg["H"] * 128), torch.zeros(2, 7, 64)
    with pytest.raises(ValueError, match="cond must be"):
        block(x, text, None, None if shape is None else torch.zeros(shape))
