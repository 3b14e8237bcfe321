"""A whole DiT block on this library: RoLA self-attention, cross-attention to a text, gated feed-forward.

    x = x + W_o  RoLA(LN(x))                    video tokens among themselves
    x = x + W_co attention(LN(x), text)         video tokens to the text tokens of their sample
    x = x + FFN(LN(x))

The norms, both attentions and the feed-forward are this library's operators with their backward passes; the
linear projections are torch's.  ``python -m paper_2609_06712_gb300.dit_block`` takes a few training steps on a
small synthetic layer and prints the loss of each.
"""
from __future__ import annotations

import torch
from torch.nn.functional import linear

from . import rola

EPS = 1e-6


class DiTBlock(torch.nn.Module):
    """One block over the token grid of a layer config (configs.py); d_model = H * 128 + the text's width d_text."""

    def __init__(self, cfg: dict, d_text: int, d_ff: int, act: str = "silu", dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.cfg, self.H, self.act = rola.make_config(cfg, rola._DTYPES[dtype]), cfg["H"], act
        d, r = self.H * 128, cfg["r"]
        made = dict(dtype=dtype, device=device)

        def weight(*shape):
            return torch.nn.Parameter(torch.randn(shape, **made) * shape[-1] ** -0.5)
        self.W_qkv, self.W_o = weight(3 * d, d), weight(d, d)
        self.W_cq, self.W_ckv, self.W_co = weight(d, d), weight(2 * d, d_text), weight(d, d)
        self.P_q, self.P_k = weight(self.H, r, 128), weight(self.H, r, 128)
        self.W_gate, self.W_up, self.W_down = weight(d_ff, d), weight(d_ff, d), weight(d, d_ff)
        self.norms = torch.nn.ParameterList(torch.nn.Parameter(t) for _ in range(3)
                                            for t in (torch.ones(d, **made), torch.zeros(d, **made)))

    def _norm(self, i, x):
        return rola.LayerNormFunction.apply(x, self.norms[2 * i], self.norms[2 * i + 1], EPS)

    def _heads(self, x, parts):
        B, N, _ = x.shape
        return x.view(B, N, parts, self.H, 128).permute(2, 0, 3, 1, 4).contiguous().unbind(0)

    def _join(self, o):
        return o.transpose(1, 2).reshape(o.shape[0], o.shape[2], self.H * 128)

    def forward(self, x, text, text_len=None):
        """x [B][N][d_model], text [B][L][d_text], text_len int32 [B] (None: the whole text)."""
        with torch.cuda.device(x.device):            # the module launches on the current device
            return self._forward(x, text, text_len)

    def _forward(self, x, text, text_len):
        q, k, v = self._heads(linear(self._norm(0, x), self.W_qkv), 3)
        x = x + linear(self._join(rola.RoLAFunction.apply(self.cfg, q, k, v, self.P_q, self.P_k, None)), self.W_o)
        (q,), (k, v) = self._heads(linear(self._norm(1, x), self.W_cq), 1), self._heads(linear(text, self.W_ckv), 2)
        x = x + linear(self._join(rola.AttentionFunction.apply(q, k, v, text_len, False)), self.W_co)
        return x + rola.FfnFunction.apply(self._norm(2, x), self.W_gate, self.W_up, self.W_down, self.act)


def train(steps: int = 5, lr: float = 0.2, seed: int = 0):
    """Losses of `steps` plain gradient steps towards a fixed random target on the tiny layer."""
    from . import configs
    torch.manual_seed(seed)
    cfg = configs.get("tiny")
    block = DiTBlock(cfg, d_text=192, d_ff=704)
    made = dict(dtype=torch.bfloat16, device="cuda")
    x, target = (torch.randn(1, cfg["N"], cfg["H"] * 128, **made) for _ in range(2))
    text, text_len = torch.randn(1, 77, 192, **made), torch.tensor([40], dtype=torch.int32, device="cuda")
    losses = []
    for _ in range(steps):
        loss = (block(x, text, text_len).float() - target.float()).square().mean()
        block.zero_grad(set_to_none=True)
        loss.backward()
        with torch.no_grad():
            for p in block.parameters():
                p.sub_(lr * p.grad)
        losses.append(loss.item())
    return losses


if __name__ == "__main__":
    for i, value in enumerate(train()):
        print(f"step {i}: loss {value:.4f}")
