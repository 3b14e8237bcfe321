"""Attention over a dense key set and its gradients on the GPU against 64-bit definitions, with the bounds of
block_util."""
import math

import pytest
import torch

from block_util import DTYPES, E, U16, U32, directional, out_u, randn, within

pytestmark = pytest.mark.gpu
D = 128


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def inputs_of(B, H, Hk, Lq, Lk, dtype, lens=None, seed=0, q_scale=1.0):
    """q, k, v, dO, kv_len.  The keys past a sequence's length hold NaN and infinity."""
    q, k, v = randn((B, H, Lq, D), dtype, seed, q_scale), randn((B, Hk, Lk, D), dtype, seed + 1), randn((B, Hk, Lk, D), dtype, seed + 2)
    dO = randn((B, H, Lq, D), dtype, seed + 3)
    if lens is None:
        return q, k, v, dO, None
    for b, n in enumerate(lens):
        if n < Lk:
            k[b, :, max(n, 0):] = float("nan")
            v[b, :, max(n, 0):] = float("inf")
    return q, k, v, dO, torch.tensor(lens, dtype=torch.int32, device="cuda")


def run(rl, causal, q, k, v, dO, kv_len, scale=0.0, backward=True):
    B, H, Lq, _ = q.shape
    c = rl.make_attention_config(B, H, k.shape[1], Lq, k.shape[2], causal, scale,
                                 rl.ROLA_BF16 if q.dtype == torch.bfloat16 else rl.ROLA_FP32)
    ws = rl.attention_workspace(c)
    o, lse = torch.full_like(q, float("nan")), torch.full((B, H, Lq), float("nan"), device="cuda")
    rl.attention(c, q, k, v, kv_len, o, lse, ws)
    assert rl.get_device_status(ws) == rl.ROLA_OK
    o2 = torch.full_like(q, float("nan"))
    rl.attention(c, q, k, v, kv_len, o2, None, ws)
    assert torch.equal(o, o2), "without lse other bits"
    if not backward:
        return o, lse
    dq, dk, dv = (torch.full_like(t, float("nan")) for t in (q, k, v))
    bws = rl.attention_backward_workspace(c)
    rl.attention_backward(c, q, k, v, kv_len, o, lse, dO, dq, dk, dv, bws)
    assert rl.get_device_status(bws) == rl.ROLA_OK
    return o, lse, dq, dk, dv


def check(causal, q, k, v, dO, kv_len, got, scale=0.0):
    B, H, Lq, _ = q.shape
    Hk, Lk = k.shape[1], k.shape[2]
    scale = scale or 1 / math.sqrt(D)
    u = out_u(q.dtype)
    r = U16 if q.dtype == torch.bfloat16 else 0.0          # p and ds as operands of the next product
    lens = [Lk] * B if kv_len is None else [min(max(int(n), 0), Lk) for n in kv_len]
    for b, n in enumerate(lens):
        for hk in range(Hk):
            dk = dv = edk = edv = 0.0
            for h in range(hk * (H // Hk), (hk + 1) * (H // Hk)):
                Q, K, V = q[b, h].double(), k[b, hk, :n].double(), v[b, hk, :n].double()
                at = f"[{b}, {h}]"
                o, lse = got[0][b, h], got[1][b, h]
                seen = torch.ones(Lq, n, dtype=torch.bool, device="cuda")
                if causal:
                    seen = seen.tril(n - Lq)
                s = (Q @ K.t() * scale).masked_fill(~seen, float("-inf"))
                empty = ~seen.any(1)
                ref_lse = torch.logsumexp(s, 1)
                p = torch.where(seen, torch.exp(s - torch.where(empty, 0.0, ref_lse)[:, None]), 0.0)
                # an absolute error of s is a relative one of p; that of lse is at most the largest of its row
                es = torch.where(seen, (D * U32 + E) * (Q.abs() @ K.abs().t()) * scale, 0.0)
                els = (es.amax(1) if n else es.sum(1)) + (n * U32 + E) * (1 + ref_lse.abs().nan_to_num(posinf=0.0))
                ep = p * (es + els[:, None] + E * (1 + s.abs().nan_to_num(posinf=0.0)))
                assert (lse[empty] == float("-inf")).all() and (o[empty] == 0).all(), f"empty rows {at}"
                within("lse " + at, lse[~empty], ref_lse[~empty], els[~empty])
                O, eO = p @ V, (ep + (n * U32 + E + r) * p) @ V.abs()
                within("o " + at, o, O, (eO + u * O.abs()) * (1 + u))
                if len(got) == 2:
                    continue
                dO_ = dO[b, h].double()
                dP, adP = dO_ @ V.t(), dO_.abs() @ V.abs().t()
                Dv = (dO_ * O).sum(1, keepdim=True)
                eD = (dO_.abs() * (eO + u * O.abs())).sum(1, keepdim=True) + (D * U32 + E) * (dO_ * O).abs().sum(1, keepdim=True)
                ds = p * (dP - Dv) * scale
                eds = (p * ((D * U32 + E) * adP + eD) + ep * (dP - Dv).abs() + (r + E) * p * (dP - Dv).abs()) * scale
                ref = ds @ K
                assert (got[2][b, h][empty] == 0).all(), f"dq of empty rows {at}"
                err = eds @ K.abs() + (n * U32 + E) * (ds.abs() @ K.abs())
                within("dq " + at, got[2][b, h], ref, (err + u * ref.abs()) * (1 + u))
                rows = Lq * (H // Hk)
                dk, edk = dk + ds.t() @ Q, edk + eds.t() @ Q.abs() + (rows * U32 + E) * (ds.abs().t() @ Q.abs())
                dv = dv + p.t() @ dO_
                edv = edv + (ep + r * p).t() @ dO_.abs() + (rows * U32 + E) * (p.t() @ dO_.abs())
            if len(got) > 2:
                at = f"[{b}, {hk}]"
                within("dk " + at, got[3][b, hk, :n], dk, (edk + u * dk.abs()) * (1 + u))
                within("dv " + at, got[4][b, hk, :n], dv, (edv + u * dv.abs()) * (1 + u))
                assert (got[3][b, hk, n:] == 0).all() and (got[4][b, hk, n:] == 0).all(), f"unseen keys {at}"


# (B, H, H_kv, Lq, Lk, causal, lens): one of everything, lengths around a tile, partial tiles, lengths of 0 and 1,
# shared heads whose rows share a row tile, causal with more keys than queries and fewer (empty rows)
CASES = [
    (1, 1, 1, 1, 1, False, None), (1, 1, 1, 1, 1, True, None), (2, 2, 1, 3, 5, False, [5, 0]),
    (1, 2, 2, 63, 65, False, None), (1, 1, 1, 64, 64, True, None), (1, 1, 1, 65, 63, True, None),
    (2, 2, 2, 127, 129, True, [129, 77]), (1, 1, 1, 128, 128, True, None), (1, 1, 1, 129, 127, False, None),
    (3, 4, 2, 130, 257, False, [257, 1, 128]), (3, 4, 2, 130, 257, True, [257, 129, 0]),
    (2, 6, 2, 1, 300, False, [300, 64]), (1, 10, 2, 1, 1000, True, None), (2, 15, 3, 7, 97, True, [97, 3]),
    (1, 4, 1, 200, 90, True, None), (2, 3, 3, 300, 513, True, [513, 300]), (1, 2, 1, 513, 700, False, None),
    (4, 2, 1, 50, 70, False, [-3, 70, 1000, 64]), (1, 2, 2, 640, 640, True, None), (1, 1, 1, 1025, 31, False, None),
]


@pytest.mark.parametrize("B,H,Hk,Lq,Lk,causal,lens", CASES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_against_64_bits(rl, B, H, Hk, Lq, Lk, causal, lens, dname):
    x = inputs_of(B, H, Hk, Lq, Lk, DTYPES[dname], lens, seed=Lq + Lk)
    check(causal, *x, run(rl, causal, *x))


# few rows over long key sets: the key axis is split
LONG = [(1, 1, 1, 1, 5000, False, None), (2, 8, 2, 1, 9001, False, [9001, 4444]), (1, 2, 2, 5, 20000, True, None),
        (3, 2, 1, 1, 3000, False, [0, 1, 3000]), (1, 5, 1, 33, 4097, False, None), (2, 2, 2, 130, 6000, True, [6000, 200])]


@pytest.mark.parametrize("B,H,Hk,Lq,Lk,causal,lens", LONG)
@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_few_rows_over_long_key_sets(rl, B, H, Hk, Lq, Lk, causal, lens, dname):
    x = inputs_of(B, H, Hk, Lq, Lk, DTYPES[dname], lens, seed=Lq + Lk)
    check(causal, *x, run(rl, causal, *x))


@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_many_heads_are_not_split(rl, dname):
    """More (head, row tile) items than SMs, one row each and many."""
    x = inputs_of(4, 48, 48, 1, 200, DTYPES[dname], [200, 13, 0, 128])
    check(False, *x, run(rl, False, *x))
    x = inputs_of(1, 20, 20, 1200, 140, DTYPES[dname])
    check(False, *x, run(rl, False, *x))


@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_scale_and_peaked_scores(rl, dname):
    """Another scale; scores of several hundred, so that the running maximum moves far and p is nearly one-hot."""
    x = inputs_of(1, 2, 1, 150, 400, DTYPES[dname], q_scale=0.5)
    check(True, *x, run(rl, True, *x, scale=0.31), scale=0.31)
    x = inputs_of(1, 2, 1, 150, 400, DTYPES[dname], q_scale=20.0)
    o, lse = run(rl, False, *x, backward=False)
    q, k, v = (t.double() for t in x[:3])
    s = q @ k.transpose(2, 3) / math.sqrt(D)
    es = (D * U32 + E) * (q.abs() @ k.abs().transpose(2, 3)).amax(3) / math.sqrt(D)
    bound = 2 * es + (400 * U32 + E) * (1 + s.abs().amax(3))
    within("lse", lse, torch.logsumexp(s, 3), bound)
    ref = torch.softmax(s, 3) @ v
    mag = torch.softmax(s, 3) @ v.abs()
    r = 2 * U16 if dname == "bf16" else 4 * U32
    within("o", o, ref, (2 * bound[..., None] + r) * mag + r * ref.abs())


def test_equal_scores_and_rising_scores(rl):
    """q = 0: the mean of the values.  Scores that rise along the keys: every tile moves the running maximum."""
    q, k, v, dO, _ = inputs_of(1, 1, 1, 70, 300, torch.bfloat16)
    o, lse = run(rl, False, q * 0, k, v, dO, None, backward=False)
    within("lse", lse, torch.full_like(lse, math.log(300)).double(), torch.full_like(lse, 1e-5).double())
    ref = v.double().mean(2, keepdim=True).expand(1, 1, 70, D)
    within("o", o, ref, U16 * 1.01 * ref.abs() + U16 * v.double().abs().mean(2, keepdim=True))
    k = torch.ones_like(k) * torch.arange(300, device="cuda").view(1, 1, 300, 1) / 64
    x = (torch.ones_like(q), k.bfloat16(), v, dO, None)
    check(False, *x, run(rl, False, *x))


@pytest.mark.parametrize("shape", [(2, 4, 2, 300, 500), (1, 8, 2, 1, 7000)])
def test_same_bits_and_streams(rl, shape):
    x = inputs_of(*shape, torch.bfloat16)
    a, b = run(rl, True, *x), run(rl, True, *x)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = run(rl, True, x[0] * 1.0, *x[1:])
    side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(a, c))


def test_gradient_against_differences(rl):
    x = list(inputs_of(2, 4, 2, 20, 45, torch.float32, seed=5))
    dO = x[3]
    o, _, *grads = run(rl, True, *x)
    scale = dO.double().norm().item() * o.double().norm().item()
    for i, grad in enumerate(grads):
        d = torch.sign(randn(x[i].shape, torch.float32, 9 + i)) * 0.25
        f = lambda t: (run(rl, True, *[t if j == i else x[j] for j in range(5)], backward=False)[0].double() * dO.double()).sum().item()  # noqa: E731
        want, gap = directional(f, x[i], d)
        assert abs((grad.double() * d.double()).sum().item() - want) <= gap + 2 * scale * 2.0 ** -20 * 2 ** 6


def test_autograd_function(rl):
    q, k, v, dO, _ = inputs_of(2, 4, 2, 40, 60, torch.float32)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    ref = [t.double().clone().requires_grad_() for t in (q, k, v)]
    rl.AttentionFunction.apply(*leaves, None, False).backward(dO)
    kk, vv = (t.repeat_interleave(2, 1) for t in ref[1:])
    (torch.softmax(ref[0] @ kk.transpose(2, 3) / math.sqrt(D), 3) @ vv).backward(dO.double())
    for a, b in zip(leaves, ref):
        assert (a.grad.double() - b.grad).norm() <= 1e-5 * b.grad.norm()


def test_refusals(rl):
    q, k, v, dO, _ = inputs_of(2, 4, 2, 8, 16, torch.bfloat16)
    c = rl.make_attention_config(2, 4, 2, 8, 16)
    ws, o = rl.attention_workspace(c), torch.empty_like(q)
    with pytest.raises(ValueError):
        rl.attention(c, q.float(), k, v, None, o, None, ws)
    with pytest.raises(ValueError):
        rl.attention(c, q, k, v[:, :1], None, o, None, ws)
    with pytest.raises(ValueError):
        rl.attention(c, q, k, v, torch.ones(2, device="cuda"), o, None, ws)
    with pytest.raises(ValueError):
        rl.attention(c, q.transpose(1, 2).contiguous().transpose(1, 2), k, v, None, o, None, ws)
    with pytest.raises(rl.RolaError):
        rl.attention(c, q, k, v, None, o, None, ws[:128])
    with pytest.raises(rl.RolaError):
        rl.attention_backward(c, q, k, v, None, o, None, dO, o, k, v, rl.attention_backward_workspace(c))
    for bad in ((2, 4, 3, 8, 16), (2, 4, 2, 0, 16), (2, 4, 2, 8, 0)):
        with pytest.raises(rl.RolaError):
            rl.attention_workspace(rl.make_attention_config(*bad))
