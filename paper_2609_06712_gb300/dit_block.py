"""A whole DiT block on this library: RoLA self-attention, cross-attention to a text, gated feed-forward.

    x = x + W_o  RoLA(LN(x))                    video tokens among themselves
    x = x + W_co attention(LN(x), text)         video tokens to the text tokens of their sample
    x = x + FFN(LN(x))

The norms, both attentions and the feed-forward are this library's operators with their backward passes; the
linear projections are torch's.  ``python -m paper_2609_06712_gb300.dit_block`` takes a few training steps on a
small synthetic layer and prints the loss of each.

With a conditioning vector (``d_cond``) the block is modulated by it, sample by sample, and its projections are this
library's too (torch's are left: the conditioning's SiLU, and the copies of q, k and v into heads and back): a linear
layer makes two shifts, scales and gates, and each branch joins the stream through its gate in the kernel that also
makes the next branch's input:

    shift_1, scale_1, gate_1, shift_2, scale_2, gate_2 = W_mod SiLU(cond) + b_mod
    y = norm(x) (1 + scale_1) + shift_1
    x, y = x + gate_1 W_o RoLA(y), norm of it
    x, y = x + W_co attention(y, text), norm of it (1 + scale_2) + shift_2
    x = x + gate_2 FFN(y)

``--conditioned`` trains that form.
"""
from __future__ import annotations

import sys

import torch
from torch.nn.functional import linear, silu

from . import rola

EPS = 1e-6


class DiTBlock(torch.nn.Module):
    """One block over the token grid of a layer config (configs.py); d_model = H * 128 + the text's width d_text;
    d_cond, if given, is the width of the conditioning vector of each sample."""

    d_cond = None                                    # width of the conditioning vector, of a conditioned block

    def __init__(self, cfg: dict, d_text: int, d_ff: int, act: str = "silu", dtype=torch.bfloat16, device="cuda",
                 d_cond: int | None = None):
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
        if d_cond is not None:
            self.d_cond = d_cond
            self.W_mod, self.b_mod = weight(6 * d, d_cond), torch.nn.Parameter(torch.zeros(6 * d, **made))

    def _norm(self, i, x):
        return rola.LayerNormFunction.apply(x, self.norms[2 * i], self.norms[2 * i + 1], EPS)

    def _heads(self, x, parts):
        B, N, _ = x.shape
        return x.view(B, N, parts, self.H, 128).permute(2, 0, 3, 1, 4).contiguous().unbind(0)

    def _join(self, o):
        return o.transpose(1, 2).reshape(o.shape[0], o.shape[2], self.H * 128)

    def forward(self, x, text, text_len=None, cond=None):
        """x [B][N][d_model], text [B][L][d_text], text_len int32 [B] (None: the whole text), cond [B][d_cond] of a
        conditioned block."""
        if (cond is None) != (self.d_cond is None) or cond is not None and cond.shape != (x.shape[0], self.d_cond):
            raise ValueError(f"DiTBlock: cond must be {'None' if self.d_cond is None else f'[B][{self.d_cond}]'}, not "
                             f"{None if cond is None else tuple(cond.shape)}")
        with torch.cuda.device(x.device):            # the module launches on the current device
            if cond is not None:
                return self._conditioned(x, text, text_len, cond)
            return self._forward(x, text, text_len)

    def _join_and_norm(self, i, x, h, gate, scale, shift):
        """x + gate h, and norm i of it, scaled and shifted."""
        return rola.ResidualNormFunction.apply(x, h, gate, None, self.norms[2 * i], self.norms[2 * i + 1], scale, shift,
                                               "layer", "none", EPS)

    def _conditioned(self, x, text, text_len, cond):
        project = rola.LinearFunction.apply          # X, W, bias, residual, activation
        mod = project(silu(cond), self.W_mod, self.b_mod, None, "identity").view(x.shape[0], 6, x.shape[2])
        shift_1, scale_1, gate_1, shift_2, scale_2, gate_2 = mod.unbind(1)
        _, y = self._join_and_norm(0, x, None, None, scale_1, shift_1)
        q, k, v = self._heads(project(y, self.W_qkv, None, None, "identity"), 3)
        h = self._join(rola.RoLAFunction.apply(self.cfg, q, k, v, self.P_q, self.P_k, None))
        x, y = self._join_and_norm(1, x, project(h, self.W_o, None, None, "identity"), gate_1, None, None)
        (q,) = self._heads(project(y, self.W_cq, None, None, "identity"), 1)
        k, v = self._heads(project(text, self.W_ckv, None, None, "identity"), 2)
        h = self._join(rola.AttentionFunction.apply(q, k, v, text_len, False))
        x, y = self._join_and_norm(2, x, project(h, self.W_co, None, None, "identity"), None, scale_2, shift_2)
        h = rola.FfnFunction.apply(y, self.W_gate, self.W_up, self.W_down, self.act)
        return rola.ResidualNormFunction.apply(x, h, gate_2, None, None, None, None, None, "none", "none", EPS)[0]

    def _forward(self, x, text, text_len):
        q, k, v = self._heads(linear(self._norm(0, x), self.W_qkv), 3)
        x = x + linear(self._join(rola.RoLAFunction.apply(self.cfg, q, k, v, self.P_q, self.P_k, None)), self.W_o)
        (q,), (k, v) = self._heads(linear(self._norm(1, x), self.W_cq), 1), self._heads(linear(text, self.W_ckv), 2)
        x = x + linear(self._join(rola.AttentionFunction.apply(q, k, v, text_len, False)), self.W_co)
        return x + rola.FfnFunction.apply(self._norm(2, x), self.W_gate, self.W_up, self.W_down, self.act)


def train(steps: int = 5, lr: float = 0.2, seed: int = 0, conditioned: bool = False):
    """Losses of `steps` plain gradient steps towards a fixed random target on the tiny layer."""
    from . import configs
    torch.manual_seed(seed)
    cfg = configs.get("tiny")
    block = DiTBlock(cfg, d_text=192, d_ff=704, d_cond=256 if conditioned else None)
    made = dict(dtype=torch.bfloat16, device="cuda")
    x, target = (torch.randn(1, cfg["N"], cfg["H"] * 128, **made) for _ in range(2))
    text, text_len = torch.randn(1, 77, 192, **made), torch.tensor([40], dtype=torch.int32, device="cuda")
    cond = torch.randn(1, 256, **made) if conditioned else None
    losses = []
    for _ in range(steps):
        loss = (block(x, text, text_len, cond).float() - target.float()).square().mean()
        block.zero_grad(set_to_none=True)
        loss.backward()
        with torch.no_grad():
            for p in block.parameters():
                p.sub_(lr * p.grad)
        losses.append(loss.item())
    return losses


if __name__ == "__main__":
    for i, value in enumerate(train(conditioned="--conditioned" in sys.argv[1:])):
        print(f"step {i}: loss {value:.4f}")
