"""Work of the operators around the attention module of a transformer block: layer norm, gated
feed-forward and softmax attention over a dense key set, forward and backward.

Each case names one operator, its sizes and its direction.  `run` computes it in a plain form
(elementary torch operations in 32 bits, rounded once at the end) where `own` is false, and through
the package's entry points where `own` is true.

Shapes: layer norm x [rows][d]; feed-forward X [tokens][d_model], W_gate, W_up [d_ff][d_model],
W_down [d_model][d_ff]; attention q [B][H][Lq][128], k, v [B][H_kv][Lk][128], kv_len int32 [B].
The widths 1536 and 5120 are 12 and 40 heads of 128, and the token counts 32760 and 75600 (or their
halves and quarters) are the 480p and 720p video layers of the package's configurations.
"""
import math
import random

import torch

own = False

HEAD = 128
LN_EPS = 1e-6


# ------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # the norm before a video layer's attention at 720p, inference: a pass over memory
        dict(name="norm 720p forward", op="norm", rows=75600, d=5120, dtype="bf16", train=False),
        # the same at the smaller 480p layer, in training: both passes and the weight's gradient
        dict(name="norm 480p training", op="norm", rows=32760, d=1536, dtype="bf16", train=True),
        # a conditioning vector's norm: one row, where a call's latency is all that counts
        dict(name="norm one row", op="norm", rows=1, d=5120, dtype="bf16", train=False),
        # a small ragged layer in 32 bits, a width that no vector load divides
        dict(name="norm odd width fp32 training", op="norm", rows=585, d=777, dtype="fp32", train=True),
        # one token through the feed-forward: every weight is read once for it
        dict(name="feed-forward one token", op="ffn", tokens=1, d_model=5120, d_ff=13824, dtype="bf16", act="silu", train=False),
        # a short prompt's tokens
        dict(name="feed-forward 77 tokens", op="ffn", tokens=77, d_model=1536, d_ff=4096, dtype="bf16", act="gelu", train=False),
        # half a 480p video at the large width, inference
        dict(name="feed-forward 16380 tokens", op="ffn", tokens=16380, d_model=5120, d_ff=13824, dtype="bf16", act="silu", train=False),
        # a quarter of a 480p video at the small width, a training step
        dict(name="feed-forward training", op="ffn", tokens=8190, d_model=1536, d_ff=4096, dtype="bf16", act="silu", train=True),
        # video tokens attending to a text: the cross-attention of the 720p layer
        dict(name="attention 720p to 512", op="attn", B=1, H=40, H_kv=40, Lq=75600, Lk=512, causal=False, ragged=0, dtype="bf16", train=False),
        # one new token for each of four sequences over long key sets of unequal lengths, heads shared
        dict(name="attention one token", op="attn", B=4, H=40, H_kv=8, Lq=1, Lk=32760, causal=False, ragged=1, dtype="bf16", train=False),
        # a causal sequence, a training step, heads shared
        dict(name="attention causal training", op="attn", B=2, H=12, H_kv=4, Lq=4095, Lk=4095, causal=True, ragged=0, dtype="bf16", train=True),
        # cross-attention to texts of unequal lengths, a training step
        dict(name="attention cross training", op="attn", B=2, H=12, H_kv=12, Lq=8190, Lk=512, causal=False, ragged=2, dtype="bf16", train=True),
    ]


def _ragged(n):
    return n + 1 if n % 128 == 0 else n         # whole tiles are among the listed cases


def _log(rng, lo, hi):
    return _ragged(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    train = rng.random() < 0.5
    op = rng.choice(["norm", "ffn", "ffn", "attn", "attn", "attn"])
    if op == "norm":
        d = rng.choice([_log(rng, 64, 5119), 8 * _log(rng, 8, 639)])
        return dict(op=op, rows=_log(rng, 1, 75600), d=d, dtype=dtype, train=train)
    if op == "ffn":
        d_model, d_ff = 8 * _log(rng, 8, 639), 8 * _log(rng, 8, 1727)
        most = 16380 if dtype == "bf16" else 2048
        most = max(1, min(most, int(1.1e12 / (d_model * d_ff * (3 if train else 1)))))
        return dict(op=op, tokens=_log(rng, 1, most), d_model=d_model, d_ff=d_ff, dtype=dtype,
                    act=rng.choice(["silu", "gelu", "relu"]), train=train)
    H_kv, group = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 3, 5])
    B, causal = rng.choice([1, 2, 3]), rng.random() < 0.4
    most = 1.2e9 if dtype == "bf16" else 2e8
    while True:
        Lk = _log(rng, 2 if train else 1, 32760)     # over one key, p is 1 and dq is 0: nothing to compare
        Lq = _ragged(max(1, Lk - rng.choice([0, 0, 1, 100, -7]))) if causal else _log(rng, 1, 16380)
        if B * H_kv * group * Lq * Lk <= most:
            break
    return dict(op=op, B=B, H=H_kv * group, H_kv=H_kv, Lq=Lq, Lk=Lk, causal=causal,
                ragged=rng.choice([0, rng.randrange(1, 1000)]), dtype=dtype, train=train)


# ---------------------------------------------------------------------------------------- inputs

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """Keys of each sequence.  Those of a ragged batch are its case's own: the first sequence has the
    whole set, the third one key or none, the others anything."""
    B, Lk = case["B"], case["Lk"]
    if not case["ragged"]:
        return [Lk] * B
    rng = random.Random(case["ragged"])
    lens = [rng.randint(0, Lk) for _ in range(B)]
    lens[0] = Lk
    if B > 2:
        lens[2] = case["ragged"] % 2
    return lens


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _dtype(case)

    def rand(*shape, scale=1.0, shift=0.0):
        return torch.empty(shape, device="cuda").normal_(shift, scale, generator=g).to(dt)

    st = dict(case=case)
    if case["op"] == "norm":
        n, d = case["rows"], case["d"]
        # a residual stream: channels of unequal size and offset
        x = torch.empty((n, d), device="cuda").normal_(generator=g)
        x = x * torch.empty((d,), device="cuda").uniform_(0.5, 3.0, generator=g)
        st["x"] = (x + torch.empty((d,), device="cuda").normal_(0.3, 0.5, generator=g)).to(dt)
        st["gamma"], st["beta"] = rand(d, scale=0.2, shift=1.0), rand(d, scale=0.2)
        if case["train"]:
            st["dy"] = rand(n, d)
    elif case["op"] == "ffn":
        m, d, f = case["tokens"], case["d_model"], case["d_ff"]
        st["X"] = rand(m, d)
        st["W_gate"], st["W_up"] = rand(f, d, scale=d ** -0.5), rand(f, d, scale=d ** -0.5)
        st["W_down"] = rand(d, f, scale=f ** -0.5)
        if case["train"]:
            st["dY"] = rand(m, d)
    else:
        B, H, Hk, Lq, Lk = (case[n] for n in ("B", "H", "H_kv", "Lq", "Lk"))
        st["q"], st["k"], st["v"] = rand(B, H, Lq, HEAD), rand(B, Hk, Lk, HEAD), rand(B, Hk, Lk, HEAD)
        st["kv_len"] = None
        if case["ragged"]:
            st["kv_len"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
            # what lies past a sequence's end is whatever was there before, and not always a number
            gone = torch.arange(Lk, device="cuda")[None, :] >= st["kv_len"][:, None]
            for n, bad in (("k", float("nan")), ("v", float("inf"))):
                st[n].masked_fill_(gone[:, None, :, None], bad)
        if case["train"]:
            st["dO"] = rand(B, H, Lq, HEAD)
    if own:
        from paper_2609_06712_gb300 import rola
        dtype = rola.ROLA_BF16 if case["dtype"] == "bf16" else rola.ROLA_FP32
        if case["op"] == "norm":
            if case["train"]:
                st["ws"] = rola.layer_norm_backward_workspace(st["x"])
        elif case["op"] == "ffn":
            c = rola.make_ffn_config(case["tokens"], case["d_model"], case["d_ff"], case["act"], dtype)
            st["cfg"], st["ws"] = c, rola.ffn_workspace(c)
            if case["train"]:
                st["bws"] = rola.ffn_backward_workspace(c)
        else:
            c = rola.make_attention_config(case["B"], case["H"], case["H_kv"], case["Lq"], case["Lk"],
                                           causal=case["causal"], dtype=dtype)
            st["cfg"], st["ws"] = c, rola.attention_workspace(c)
            if case["train"]:
                st["bws"] = rola.attention_backward_workspace(c)
    return st


# ------------------------------------------------------------------------------------------- run

def run(state):
    return {"norm": _norm, "ffn": _ffn, "attn": _attn}[state["case"]["op"]](state)


def _norm(st):
    x, gamma, beta, train = st["x"], st["gamma"], st["beta"], st["case"]["train"]
    n, d = x.shape
    if own:
        from paper_2609_06712_gb300 import rola
        y = torch.empty_like(x)
        if not train:
            rola.layer_norm(x, gamma, beta, LN_EPS, y)
            return dict(y=y)
        mean, rstd = (torch.empty((n,), dtype=torch.float32, device=x.device) for _ in range(2))
        dgamma, dbeta = (torch.empty((d,), dtype=torch.float32, device=x.device) for _ in range(2))
        dx = torch.empty_like(x)
        rola.layer_norm(x, gamma, beta, LN_EPS, y, mean, rstd)
        rola.layer_norm_backward(x, gamma, mean, rstd, st["dy"], dx, dgamma, dbeta, st["ws"])
        return dict(y=y, dx=dx, dgamma=dgamma, dbeta=dbeta)
    xf, gf = x.float(), gamma.float()
    mean = xf.mean(dim=1, keepdim=True)
    xc = xf - mean
    rstd = torch.rsqrt((xc * xc).mean(dim=1, keepdim=True) + LN_EPS)
    xh = xc * rstd
    y = (xh * gf + beta.float()).to(x.dtype)
    if not train:
        return dict(y=y)
    dy = st["dy"].float()
    a = dy * gf
    dx = rstd * (a - a.mean(dim=1, keepdim=True) - xh * (a * xh).mean(dim=1, keepdim=True))
    return dict(y=y, dx=dx.to(x.dtype), dgamma=(dy * xh).sum(dim=0), dbeta=dy.sum(dim=0))


def _act(name, g):
    """phi(g) and phi'(g) of the gate."""
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))


def _ffn(st):
    case, X = st["case"], st["X"]
    Wg, Wu, Wd = st["W_gate"], st["W_up"], st["W_down"]
    if own:
        from paper_2609_06712_gb300 import rola
        c, Y = st["cfg"], torch.empty_like(X)
        if not case["train"]:
            rola.ffn(c, X, Wg, Wu, Wd, Y, st["ws"])
            return dict(Y=Y)
        G, U = (torch.empty((case["tokens"], case["d_ff"]), dtype=torch.float32, device=X.device) for _ in range(2))
        dX, dWg, dWu, dWd = (torch.empty_like(t) for t in (X, Wg, Wu, Wd))
        rola.ffn_train(c, X, Wg, Wu, Wd, Y, G, U, st["ws"])
        rola.ffn_backward(c, X, Wg, Wu, Wd, G, U, st["dY"], dX, dWg, dWu, dWd, st["bws"])
        return dict(Y=Y, dX=dX, dW_gate=dWg, dW_up=dWu, dW_down=dWd)
    Xf, Wgf, Wuf, Wdf = (t.float() for t in (X, Wg, Wu, Wd))
    G, U = Xf @ Wgf.t(), Xf @ Wuf.t()
    a, da = _act(case["act"], G)
    H = a * U
    Y = (H @ Wdf.t()).to(X.dtype)
    if not case["train"]:
        return dict(Y=Y)
    dY = st["dY"].float()
    dH = dY @ Wdf
    dG, dU = dH * U * da, dH * a
    out = dict(dX=dG @ Wgf + dU @ Wuf, dW_gate=dG.t() @ Xf, dW_up=dU.t() @ Xf, dW_down=dY.t() @ H)
    return dict(Y=Y, **{n: t.to(X.dtype) for n, t in out.items()})


def _attn(st):
    case, q, k, v, kv_len = st["case"], st["q"], st["k"], st["v"], st["kv_len"]
    B, H, Hk, Lq, Lk = (case[n] for n in ("B", "H", "H_kv", "Lq", "Lk"))
    if own:
        from paper_2609_06712_gb300 import rola
        c, o = st["cfg"], torch.empty_like(q)
        if not case["train"]:
            rola.attention(c, q, k, v, kv_len, o, None, st["ws"])
            return dict(o=o)
        lse = torch.empty((B, H, Lq), dtype=torch.float32, device=q.device)
        dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
        rola.attention(c, q, k, v, kv_len, o, lse, st["ws"])
        rola.attention_backward(c, q, k, v, kv_len, o, lse, st["dO"], dq, dk, dv, st["bws"])
        return dict(o=o, dq=dq, dk=dk, dv=dv)
    G, scale = H // Hk, HEAD ** -0.5
    # the heads that share a key set are more rows over it
    qf = q.float().view(B, Hk, G * Lq, HEAD)
    lens = torch.full((B,), Lk, device=q.device) if kv_len is None else kv_len
    j = torch.arange(Lk, device=q.device)
    seen = (j[None, :] < lens[:, None])[:, None, None, :]
    kf, vf = (torch.where(seen.transpose(2, 3), t.float(), 0.0) for t in (k, v))
    if case["causal"]:
        # query i of Lq stands at key position i + len - Lq
        at = torch.arange(Lq, device=q.device).repeat(G)[None, :] + (lens[:, None] - Lq)
        seen = seen & (j[None, None, None, :] <= at[:, None, :, None])
    s = qf @ kf.transpose(2, 3)
    s.mul_(scale).masked_fill_(~seen, float("-inf"))
    m = s.amax(dim=3, keepdim=True).clamp_(min=-3e38)
    p = s.sub_(m).exp_()
    l = p.sum(dim=3, keepdim=True)
    p.mul_(torch.where(l > 0, 1 / l, 0.0))
    of = p @ vf
    o = of.view(B, H, Lq, HEAD).to(q.dtype)
    if not case["train"]:
        return dict(o=o)
    dO = st["dO"].float().view(B, Hk, G * Lq, HEAD)
    dv = p.transpose(2, 3) @ dO
    ds = dO @ vf.transpose(2, 3)
    ds.sub_((dO * of).sum(dim=3, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = ds @ kf, ds.transpose(2, 3) @ qf
    return dict(o=o, dq=dq.view_as(q).to(q.dtype), dk=dk.to(q.dtype), dv=dv.to(q.dtype))


# ------------------------------------------------------------------------------------------ floor

def _pairs(case):
    """Query-key pairs that see each other, over all heads."""
    Lq, total = case["Lq"], 0
    for n in _lengths(case):
        if not case["causal"]:
            total += Lq * n
        else:                                   # query i sees max(0, i + n - Lq + 1) keys
            rows = min(Lq, n)
            total += rows * (2 * n - rows + 1) // 2
    return case["H"] * total


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        n, d = case["rows"], case["d"]
        if not case["train"]:
            return dict(bytes=2 * n * d * e + 2 * d * e, flops=8 * n * d)
        return dict(bytes=4 * n * d * e + 2 * d * e + 2 * d * 4, flops=20 * n * d)
    if case["op"] == "ffn":
        m, d, f = case["tokens"], case["d_model"], case["d_ff"]
        if not case["train"]:
            return dict(bytes=e * (2 * m * d + 3 * d * f), flops=6 * m * d * f)
        return dict(bytes=e * (4 * m * d + 6 * d * f), flops=18 * m * d * f)
    # k and v are read up to each sequence's length; their gradients are written whole
    rows, keys = case["B"] * case["H"] * case["Lq"], case["H_kv"] * sum(_lengths(case))
    if not case["train"]:
        return dict(bytes=e * HEAD * 2 * (rows + keys), flops=4 * HEAD * _pairs(case))
    whole = case["B"] * case["H_kv"] * case["Lk"]
    return dict(bytes=e * HEAD * (4 * rows + 2 * keys + 2 * whole), flops=14 * HEAD * _pairs(case))


# ------------------------------------------------------------------------------------------ exact

def exact(case, seed):
    """The same from the definitions, in 64 bits."""
    if work(case)["flops"] > 1.0e13:
        return None
    st = {n: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() else t
          for n, t in prepare(case, seed).items()}
    return {"norm": _norm64, "ffn": _ffn64, "attn": _attn64}[case["op"]](case, st)


def _norm64(case, st):
    out = {n: [] for n in ("y", "dx")}
    dgamma = dbeta = 0.0
    for lo in range(0, case["rows"], 16384):
        x = st["x"][lo:lo + 16384]
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        sigma = (var + LN_EPS).sqrt()
        xh = (x - mean) / sigma
        out["y"].append(xh * st["gamma"] + st["beta"])
        if case["train"]:
            dy = st["dy"][lo:lo + 16384]
            dxh = dy * st["gamma"]
            # the Jacobian (I - 1 1^T / d - xh xh^T / d) / sigma
            out["dx"].append((dxh - dxh.sum(1, keepdim=True) / case["d"]
                              - xh * ((dxh * xh).sum(1, keepdim=True) / case["d"])) / sigma)
            dgamma, dbeta = dgamma + (dy * xh).sum(0), dbeta + dy.sum(0)
    if not case["train"]:
        return dict(y=torch.cat(out["y"]))
    return dict(y=torch.cat(out["y"]), dx=torch.cat(out["dx"]), dgamma=dgamma, dbeta=dbeta)


def _ffn64(case, st):
    names = ("X", "W_gate", "W_up", "W_down")
    leaves = [st[n].requires_grad_(case["train"]) for n in names]
    X, Wg, Wu, Wd = leaves
    with torch.set_grad_enabled(case["train"]):
        g = torch.nn.functional.linear(X, Wg)
        if case["act"] == "silu":
            a = g / (1 + torch.exp(-g))
        elif case["act"] == "relu":
            a = g.clamp(min=0)
        else:
            a = g * torch.special.ndtr(g)
        Y = torch.nn.functional.linear(a * torch.nn.functional.linear(X, Wu), Wd)
    if not case["train"]:
        return dict(Y=Y)
    grads = torch.autograd.grad(Y, leaves, st["dY"])
    return dict(Y=Y.detach(), **{"d" + n: t for n, t in zip(names, grads)})


def _attn64(case, st):
    B, H, Hk, Lq, Lk = (case[n] for n in ("B", "H", "H_kv", "Lq", "Lk"))
    q, k, v = st["q"], st["k"], st["v"]
    o = torch.zeros_like(q)
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    for b in range(B):
        n = Lk if st["kv_len"] is None else int(st["kv_len"][b])
        # rows that see a key at all: with a causal mask query i sees the keys up to i + n - Lq
        lo = max(0, Lq - n) if case["causal"] else 0
        if n == 0 or lo >= Lq:
            continue
        hidden = None
        if case["causal"]:
            hidden = torch.ones(Lq, n, dtype=torch.bool, device=q.device).triu(n - Lq + 1)[lo:]
        for h in range(H):
            hk = h // (H // Hk)
            for r0 in range(lo, Lq, 8192):
                r1 = min(Lq, r0 + 8192)
                qs, ks, vs = q[b, h, r0:r1], k[b, hk, :n], v[b, hk, :n]
                w = (qs @ ks.t()) / math.sqrt(HEAD)
                if hidden is not None:
                    w.masked_fill_(hidden[r0 - lo:r1 - lo], float("-inf"))
                w = torch.softmax(w, dim=1)
                o[b, h, r0:r1] = w @ vs
                if case["train"]:
                    dO = st["dO"][b, h, r0:r1]
                    dw = dO @ vs.t()
                    dw = w * (dw - (w * dw).sum(1, keepdim=True)) / math.sqrt(HEAD)
                    grads[0][b, h, r0:r1] = dw @ ks
                    grads[1][b, hk, :n] += dw.t() @ qs
                    grads[2][b, hk, :n] += w.t() @ dO
    if not case["train"]:
        return dict(o=o)
    return dict(o=o, dq=grads[0], dk=grads[1], dv=grads[2])
