"""Dense attention where every CTA takes items of several turns, without a split: causal (the turns run forwards and
backwards over items sorted by length), shared heads whose rows wrap within a tile, ragged."""
import pytest
import torch

import test_attention_gpu as base
from block_util import DTYPES

pytestmark = pytest.mark.gpu
rl = base.rl


@pytest.mark.parametrize("B,H,Hk,Lq,Lk,causal,lens", [
    (2, 48, 48, 1100, 1100, True, None), (1, 80, 20, 900, 900, True, None), (3, 60, 30, 500, 470, True, [470, 200, 1]),
    (4, 40, 40, 600, 300, False, [300, 129, 64, 0]), (2, 120, 40, 333, 700, True, None)])
def test_items_of_several_turns(rl, B, H, Hk, Lq, Lk, causal, lens):
    c = rl.make_attention_config(B, H, Hk, Lq, Lk, causal)
    rows = H // Hk * Lq
    assert B * Hk * -(-rows // 256) > 152
    # no parts: the status alone forward, D beside it backward
    assert rl.attention_workspace(c).numel() == 256
    assert rl.attention_backward_workspace(c).numel() == 256 + -(-4 * B * H * Lq // 256) * 256
    x = base.inputs_of(B, H, Hk, Lq, Lk, DTYPES["bf16"], lens, seed=Lq)
    got = base.run(rl, causal, *x)
    base.check(causal, *x, got)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(base.run(rl, causal, *x), got))
