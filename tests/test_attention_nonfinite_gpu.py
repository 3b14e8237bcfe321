"""Attention over NaN and infinite queries and keys that are seen: o and lse are NaN exactly where the definition's are,
whether the key axis is split or not, and the other rows are untouched."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def tensors(B, H, Hk, Lq, Lk, dt):
    g = torch.Generator().manual_seed(Lq + Lk)
    return [torch.randn(s, generator=g).to(dt).cuda() for s in ((B, H, Lq, 128), (B, Hk, Lk, 128), (B, Hk, Lk, 128))]


def run(rl, q, k, v, causal=False, lens=None):
    B, H, Lq, _ = q.shape
    code = rl.ROLA_BF16 if q.dtype == torch.bfloat16 else rl.ROLA_FP32
    c = rl.make_attention_config(B, H, k.shape[1], Lq, k.shape[2], causal, dtype=code)
    o, lse, ws = torch.full_like(q, 7.0), torch.full((B, H, Lq), 7.0, device="cuda"), rl.attention_workspace(c)
    kv = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    rl.attention(c, q, k, v, kv, o, lse, ws)
    assert rl.get_device_status(ws) == rl.ROLA_OK
    return o, lse


def definition(q, k, v, causal=False, lens=None):
    B, H, Lq, _ = q.shape
    Hk, Lk = k.shape[1], k.shape[2]
    kk, vv = (t.double().repeat_interleave(H // Hk, 1) for t in (k, v))
    n = torch.tensor([Lk] * B if lens is None else lens, device="cuda").view(B, 1, 1, 1)
    j, i = torch.arange(Lk, device="cuda"), torch.arange(Lq, device="cuda").view(Lq, 1)
    seen = (j < n) & ((j <= i + n - Lq) if causal else torch.ones((), dtype=torch.bool, device="cuda"))
    s = (q.double() @ kk.transpose(2, 3) / math.sqrt(128)).masked_fill(~seen, float("-inf"))
    p = torch.softmax(s, 3).masked_fill(~seen, 0.0)              # of an empty row: 0
    vv = torch.where((j < n).transpose(2, 3), vv, 0.0)
    # about the row's maximum: inf - inf where that is infinite
    lse = torch.where((s == float("inf")).any(3), float("nan"), torch.logsumexp(s, 3))
    return p @ vv, lse


def check(got, want):
    (o, lse), (ref, ref_lse) = got, want
    assert torch.equal(torch.isnan(o), torch.isnan(ref)) and torch.equal(torch.isnan(lse), torch.isnan(ref_lse))
    good = ~torch.isnan(ref)
    # P rounded to bf16 (2^-8 of values that average to |o| or less: |v| is below 6) and o once more
    tol = 0.06 if o.dtype == torch.bfloat16 else 1e-4
    assert ((o.double() - ref)[good].abs() <= tol).all()
    fin = torch.isfinite(ref_lse)
    assert torch.equal(lse[~fin & ~torch.isnan(ref_lse)].double(), ref_lse[~fin & ~torch.isnan(ref_lse)])
    assert ((lse.double() - ref_lse)[fin].abs() <= 1e-3).all()


# one part, parts of a split key axis, and a batch whose second sequence fits one part
SHAPES = [(1, 2, 2, 3, 100, False, None), (1, 3, 1, 300, 400, True, None), (1, 2, 2, 1, 6000, False, None),
          (2, 4, 2, 2, 5000, True, [5000, 90]), (2, 2, 1, 1, 4000, False, [0, 4000])]


@pytest.mark.parametrize("B,H,Hk,Lq,Lk,causal,lens", SHAPES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_queries(rl, B, H, Hk, Lq, Lk, causal, lens, dname, bad):
    q, k, v = tensors(B, H, Hk, Lq, Lk, DTYPES[dname])
    q[B - 1, 0, Lq - 1, 5] = bad
    check(run(rl, q, k, v, causal, lens), definition(q, k, v, causal, lens))
    # every score of the row -inf: 0 / 0
    k[..., 5] = torch.where(k[..., 5] == 0, 1.0, k[..., 5].abs())
    q[B - 1, 0, Lq - 1, 5] = float("-inf")
    check(run(rl, q, k, v, causal, lens), definition(q, k, v, causal, lens))


@pytest.mark.parametrize("B,H,Hk,Lq,Lk,causal,lens", SHAPES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("at", [0, 60, -1])
def test_keys(rl, B, H, Hk, Lq, Lk, causal, lens, dname, at):
    q, k, v = tensors(B, H, Hk, Lq, Lk, DTYPES[dname])
    n = Lk if lens is None else lens[-1]
    for bad in (float("nan"), float("inf")):
        k[B - 1, 0, at % n, 7] = bad
        check(run(rl, q, k, v, causal, lens), definition(q, k, v, causal, lens))


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("first", [64, 65, 128, 200])
def test_a_row_whose_first_scores_are_minus_infinity(rl, dname, first):
    """Finite scores far below 0 after whole steps of -inf: the running maximum has to start with them."""
    q, k, v = tensors(1, 2, 1, 130, 300, DTYPES[dname])
    q.zero_()
    q[..., 3], q[..., 10] = 1.0, 8.0
    k[..., 10] -= 200.0                              # scores of -140: 2^-200 of what a maximum of 0 would ask for
    k[:, :, :first, 3] = float("-inf")
    check(run(rl, q, k, v), definition(q, k, v))


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("B,H,Hk,Lq,Lk,lens", [(1, 4, 2, 300, 200, None), (2, 6, 2, 170, 160, [160, 140]), (1, 2, 1, 90, 60, None)])
def test_dq_of_queries_that_see_nothing(rl, dname, B, H, Hk, Lq, Lk, lens):
    """It is 0 whatever the incoming gradient holds there: rows in front of a causal sequence, beside the last rows of
    the head before in the same tile."""
    q, k, v = tensors(B, H, Hk, Lq, Lk, DTYPES[dname])
    code = rl.ROLA_BF16 if dname == "bf16" else rl.ROLA_FP32
    c = rl.make_attention_config(B, H, Hk, Lq, Lk, True, dtype=code)
    kv = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((B, H, Lq), device="cuda")
    rl.attention(c, q, k, v, kv, o, lse, rl.attention_workspace(c))
    dO = torch.randn(q.shape, generator=torch.Generator().manual_seed(1)).to(q.dtype).cuda()
    clean, grads = ([torch.empty_like(t) for t in (q, k, v)] for _ in range(2))
    bws = rl.attention_backward_workspace(c)
    rl.attention_backward(c, q, k, v, kv, o, lse, dO, *clean, bws)
    empty = [Lq - n for n in (lens or [Lk] * B)]
    for b, n in enumerate(empty):
        dO[b, :, :n, 3] = float("inf")
        dO[b, :, :n, 40] = float("nan")
    rl.attention_backward(c, q, k, v, kv, o, lse, dO, *grads, bws)
    for b, n in enumerate(empty):
        assert (grads[0][b, :, :n] == 0).all() and torch.equal(grads[0][b, :, n:], clean[0][b, :, n:])
