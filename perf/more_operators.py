"""Work of the operators that join the parts of a conditioned transformer block: linear layers with bias, activation and
residual, and the gated residual sum with the norms before and after it, forward and backward.

Each case names one operator, its sizes and its direction.  `run` computes it in a plain form
(elementary torch operations in 32 bits, rounded once at the end) where `own` is false, and through
the package's entry points where `own` is true.

Shapes: linear X [tokens][d_in], W [d_out][d_in], b [d_out], residual [tokens][d_out]; residual norm
x, h [groups][rows][d], gate, scale, shift [groups][d] (slices of one modulation [groups][6 d]), gamma, beta, gamma_h [d].
The widths 1536 and 5120 are 12 and 40 heads of 128, and the token counts 32760 and 75600 (or their
halves and quarters) are the 480p and 720p video layers of the package's configurations.
"""
import math
import random

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------------------------------ cases

def _linear(name, tokens, d_in, d_out, act, residual, dtype="bf16", train=False):
    return dict(name=name, op="linear", tokens=tokens, d_in=d_in, d_out=d_out, act=act, residual=residual, dtype=dtype,
                train=train)


def _norm(name, groups, rows, d, norm, branch, affine, mod, dtype="bf16", train=False):
    return dict(name=name, op="norm", groups=groups, rows=rows, d=d, norm=norm, branch=branch, affine=affine, mod=mod,
                dtype=dtype, train=train)


def listed():
    return [
        # a diffusion step's time through the first layer of its embedding: a call's latency is all that counts
        _linear("linear time embedding", 1, 256, 1536, "silu", False),
        # the modulation vectors of one block for two samples: every weight is read once for them
        _linear("linear modulation", 2, 5120, 30720, "identity", False),
        # the text tokens of two samples into the model's width
        _linear("linear text embedding", 514, 4096, 5120, "gelu", False),
        # the projection behind an attention onto the residual stream, a whole 720p video, inference
        _linear("linear 720p projection", 75600, 5120, 5120, "identity", True),
        # the first layer of an ungated feed-forward, a quarter of a 480p video, a training step
        _linear("linear gelu training", 8190, 1536, 6144, "gelu", False, train=True),
        # the projection behind an attention at 480p, a training step: few weights, many tokens
        _linear("linear 480p training", 32760, 1536, 1536, "identity", True, train=True),
        # a small ragged layer in 32 bits
        _linear("linear fp32 training", 585, 776, 1000, "tanh", False, dtype="fp32", train=True),
        # one token between two blocks of a wide model, where latency counts
        _norm("residual norm one token", 1, 1, 5120, "rms", "none", True, False),
        # between two blocks of the 720p layer, conditioned by its sample, inference: a pass over memory
        _norm("residual norm 720p", 1, 75600, 5120, "layer", "none", False, True),
        # the same for two half videos at 480p, a training step
        _norm("residual norm 480p training", 2, 16380, 1536, "layer", "none", False, True, train=True),
        # a block whose branch has a norm behind it too, ragged samples, a training step
        _norm("residual norm sandwich", 3, 4095, 2560, "rms", "rms", True, True, train=True),
        # every vector there is, 32 bits, a width that no vector load divides
        _norm("residual norm odd fp32", 3, 195, 777, "layer", "layer", True, True, dtype="fp32", train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = "fp32" if rng.random() < 0.2 else "bf16"
    train = rng.random() < 0.5
    if rng.random() < 0.5:
        d_in, d_out = 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 2048)
        most = 1.9e12 if dtype == "bf16" else 3e10
        most = max(1, min(32760 if dtype == "bf16" else 2048, int(most / (d_in * d_out * (3 if train else 1)))))
        # (relu's gradient jumps at 0, where the sign of a sum near it is any rounding's: inference only)
        acts = ["identity", "identity", "silu", "gelu", "tanh"] + ([] if train else ["relu"])
        c = _linear("", _log(rng, 1, most), d_in, d_out, rng.choice(acts), rng.random() < 0.5, dtype, train)
    else:
        groups = rng.choice([1, 1, 2, 3, 5, 16])
        rows = max(1, _log(rng, groups, 75600) // groups)
        d = rng.choice([_log(rng, 64, 5119), 8 * _log(rng, 8, 639), 8 * _log(rng, 8, 639)])
        c = _norm("", groups, rows, d, rng.choice(["layer", "rms"]), rng.choice(["none", "none", "layer", "rms"]),
                  rng.random() < 0.5, rng.random() < 0.7, dtype, train)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def rand(*shape, scale=1.0, shift=0.0):
        return torch.empty(shape, device="cuda").normal_(shift, scale, generator=g).to(dt)

    st = dict(case=case)
    if case["op"] == "linear":
        m, k, n = case["tokens"], case["d_in"], case["d_out"]
        st["X"], st["W"], st["b"] = rand(m, k), rand(n, k, scale=k ** -0.5), rand(n, scale=0.2)
        st["residual"] = rand(m, n) if case["residual"] else None
        if case["train"]:
            st["dY"] = rand(m, n)
    else:
        B, n, d = case["groups"], case["rows"], case["d"]
        # a residual stream: channels of unequal size and offset
        x = torch.empty((B, n, d), device="cuda").normal_(generator=g)
        x = x * torch.empty((d,), device="cuda").uniform_(0.5, 3.0, generator=g)
        st["x"] = (x + torch.empty((d,), device="cuda").normal_(0.3, 0.5, generator=g)).to(dt)
        st["h"] = rand(B, n, d)
        # one modulation of six vectors a sample, as a linear layer makes it; the block uses three of them here
        st["mod"] = rand(B, 6, d, scale=0.5)
        st["gate"], st["scale"], st["shift"] = st["mod"][:, 2], None, None
        if case["mod"]:
            st["shift"], st["scale"] = st["mod"][:, 3], st["mod"][:, 4]
        st["gamma"] = rand(d, scale=0.2, shift=1.0) if case["affine"] else None
        st["beta"] = rand(d, scale=0.2) if case["affine"] and case["norm"] == "layer" else None
        st["gamma_h"] = rand(d, scale=0.2, shift=1.0) if case["branch"] != "none" else None
        if case["train"]:
            st["dout"], st["dy"] = rand(B, n, d), rand(B, n, d)
    if own:
        from paper_2609_06712_gb300 import rola
        dtype = rola.ROLA_BF16 if case["dtype"] == "bf16" else rola.ROLA_FP32
        if case["op"] == "linear":
            c = rola.make_linear_config(case["tokens"], case["d_in"], case["d_out"], case["act"], dtype)
            st["cfg"], st["ws"] = c, rola.linear_workspace(c)
            if case["train"]:
                st["bws"] = rola.linear_backward_workspace(c)
        else:
            c = rola.make_residual_norm_config(case["groups"], case["rows"], case["d"], case["norm"], case["branch"],
                                               EPS, mod_stride=6 * case["d"], dtype=dtype)
            st["cfg"] = c
            if case["train"]:
                st["bws"] = rola.residual_norm_backward_workspace(c)
    return st


# ------------------------------------------------------------------------------------------- run

def run(state):
    return (_run_linear if state["case"]["op"] == "linear" else _run_norm)(state)


def _act(name, z):
    """phi(z) and phi'(z)."""
    if name == "identity":
        return z, torch.ones_like(z)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if name == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on
    if name == "tanh":
        t = torch.tanh(z)
        return t, 1 - t * t
    cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
    return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _run_linear(st):
    case, X, W, b, R = st["case"], st["X"], st["W"], st["b"], st["residual"]
    m, n = case["tokens"], case["d_out"]
    if own:
        from paper_2609_06712_gb300 import rola
        c, Y = st["cfg"], torch.empty((m, n), dtype=X.dtype, device=X.device)
        if not case["train"]:
            rola.linear(c, X, W, b, R, Y, st["ws"])
            return dict(Y=Y)
        Z = None                                  # the identity's gradient needs no argument
        if case["act"] != "identity":
            Z = torch.empty((m, n), dtype=torch.float32, device=X.device)
        dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty((n,), dtype=torch.float32, device=X.device)
        rola.linear_train(c, X, W, b, R, Y, Z, st["ws"])
        rola.linear_backward(c, X, W, Z, st["dY"], dX, dW, db, st["bws"])
        return dict(Y=Y, dX=dX, dW=dW, db=db)
    Xf, Wf = X.float(), W.float()
    Z = Xf @ Wf.t() + b.float()
    a, da = _act(case["act"], Z)
    Y = (a if R is None else a + R.float()).to(X.dtype)
    if not case["train"]:
        return dict(Y=Y)
    dZ = st["dY"].float() * da
    return dict(Y=Y, dX=(dZ @ Wf).to(X.dtype), dW=(dZ.t() @ Xf).to(X.dtype), db=dZ.sum(dim=0))


def _plain_norm(kind, v):
    """The normalised rows and 1 / their size."""
    c = v - v.mean(dim=-1, keepdim=True) if kind == "layer" else v
    r = torch.rsqrt((c * c).mean(dim=-1, keepdim=True) + EPS)
    return c * r, r


def _norm_grad(kind, a, vh, r):
    """From the gradient of the normalised rows to that of the rows."""
    g = a - vh * (a * vh).mean(dim=-1, keepdim=True)
    return r * (g - a.mean(dim=-1, keepdim=True) if kind == "layer" else g)


def _run_norm(st):
    case, x, h = st["case"], st["x"], st["h"]
    gate, scale, shift, gamma, beta, gamma_h = (st[n] for n in ("gate", "scale", "shift", "gamma", "beta", "gamma_h"))
    B, n, d = x.shape
    if own:
        from paper_2609_06712_gb300 import rola
        c, out, y = st["cfg"], torch.empty_like(x), torch.empty_like(x)
        vectors = dict(gate=gate, gamma_h=gamma_h, gamma=gamma, beta=beta, scale=scale, shift=shift)
        if not case["train"]:
            rola.residual_norm(c, x, h, out, y, **vectors)
            return dict(out=out, y=y)
        del vectors["shift"]

        def f32(like, *shape):
            return None if like is None else torch.empty(shape, dtype=torch.float32, device=x.device)
        stats = torch.empty((B, n, 4), dtype=torch.float32, device=x.device)
        dx, dh = torch.empty_like(x), torch.empty_like(h)
        grads = dict(dgate=f32(gate, B, d), dgamma_h=f32(gamma_h, d), dgamma=f32(gamma, d), dbeta=f32(beta, d),
                     dscale=f32(scale, B, d), dshift=f32(shift, B, d))
        rola.residual_norm(c, x, h, out, y, shift=shift, stats=stats, **vectors)
        rola.residual_norm_backward(c, x, h, stats, st["dout"], st["dy"], dx, dh, st["bws"], **vectors, **grads)
        return dict(out=out, y=y, dx=dx, dh=dh, **{k: t for k, t in grads.items() if t is not None})
    hf, one = h.float(), torch.ones((), device=x.device)
    hh, rh = (hf, None) if case["branch"] == "none" else _plain_norm(case["branch"], hf)
    wh = one if gamma_h is None else gamma_h.float()
    g = gate.float()[:, None]
    u = x.float() + g * (hh * wh)
    xh, r = _plain_norm(case["norm"], u)
    w = one if gamma is None else gamma.float()
    affine = xh * w if beta is None else xh * w + beta.float()
    s1 = one if scale is None else 1 + scale.float()[:, None]
    y = affine * s1 if shift is None else affine * s1 + shift.float()[:, None]
    out = dict(out=u.to(x.dtype), y=y.to(x.dtype))
    if not case["train"]:
        return out
    dy = st["dy"].float()
    t = st["dout"].float() + _norm_grad(case["norm"], dy * (s1 * w), xh, r)
    e = t * (g * wh)
    dh = e if case["branch"] == "none" else _norm_grad(case["branch"], e, hh, rh)
    out.update(dx=t.to(x.dtype), dh=dh.to(x.dtype), dgate=(t * hh * wh).sum(dim=1))
    if gamma_h is not None:
        out["dgamma_h"] = (t * hh * g).sum(dim=(0, 1))
    if gamma is not None:
        out["dgamma"] = (dy * xh * s1).sum(dim=(0, 1))
    if beta is not None:
        out["dbeta"] = (dy * s1).sum(dim=(0, 1))
    if scale is not None:
        out.update(dscale=(dy * affine).sum(dim=1), dshift=dy.sum(dim=1))
    return out


# ------------------------------------------------------------------------------------------ floor

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "linear":
        m, k, n = case["tokens"], case["d_in"], case["d_out"]
        plain = m * k + n * k + n + m * n * (2 if case["residual"] else 1)
        if not case["train"]:
            return dict(bytes=e * plain, flops=2 * m * n * k)
        return dict(bytes=e * (plain + m * n + m * k + n * k) + 4 * n, flops=6 * m * n * k)
    B, n, d = case["groups"], case["rows"], case["d"]
    of_group = 1 + (2 if case["mod"] else 0)
    of_all = (1 if case["branch"] != "none" else 0) + ((2 if case["norm"] == "layer" else 1) if case["affine"] else 0)
    vectors = (of_group * B + of_all) * d
    if not case["train"]:
        return dict(bytes=e * (4 * B * n * d + vectors), flops=10 * B * n * d)
    return dict(bytes=e * (8 * B * n * d + vectors) + 4 * vectors, flops=30 * B * n * d)


# ------------------------------------------------------------------------------------------ exact

def exact(case, seed):
    """The same from the definitions, in 64 bits; gradients by differentiating them."""
    if work(case)["flops"] > 1.0e13:
        return None
    st = {n: t.double() if isinstance(t, torch.Tensor) and t.is_floating_point() and n != "mod" else t
          for n, t in prepare(case, seed).items()}
    return (_linear64 if case["op"] == "linear" else _norm64)(case, st)


def _linear64(case, st):
    acts = dict(identity=lambda z: z, silu=lambda z: z / (1 + torch.exp(-z)), relu=lambda z: z.clamp(min=0),
                tanh=torch.tanh, gelu=lambda z: z * torch.special.ndtr(z))
    leaves = [st[n].requires_grad_(case["train"]) for n in ("X", "W", "b")]
    with torch.set_grad_enabled(case["train"]):
        Y = acts[case["act"]](torch.addmm(leaves[2], leaves[0], leaves[1].t()))
    whole = Y.detach() if st["residual"] is None else Y.detach() + st["residual"]
    if not case["train"]:
        return dict(Y=whole)
    return dict(Y=whole, **dict(zip(("dX", "dW", "db"), torch.autograd.grad(Y, leaves, st["dY"]))))


def _norm64(case, st):
    def normal(kind, v):
        if kind == "layer":
            var, mean = torch.var_mean(v, dim=-1, unbiased=False, keepdim=True)
            return (v - mean) / (var + EPS).sqrt()
        return v / (v.square().mean(dim=-1, keepdim=True) + EPS).sqrt()

    def sample(x, h, gate, scale, shift):
        branch = h if case["branch"] == "none" else normal(case["branch"], h) * st["gamma_h"]
        u = x + branch * gate
        y = normal(case["norm"], u)
        if st["gamma"] is not None:
            y = y * st["gamma"]
        if st["beta"] is not None:
            y = y + st["beta"]
        return u, y if scale is None else y * (1 + scale) + shift

    names = ["x", "h", "gate"] + (["scale", "shift"] if case["mod"] else [])
    shared = [n for n in ("gamma_h", "gamma", "beta") if st[n] is not None]
    out = {}
    for i in range(case["groups"]):
        rows = {n: [] for n in ("out", "y", "x", "h")}
        sums = {}
        step = max(1, (1 << 27) // case["d"])                    # rows at a time: 1 GB a tensor
        for lo in range(0, case["rows"], step):
            part = {n: st[n][i, lo:lo + step] if n in ("x", "h") else st[n][i] for n in names}
            leaves = [part[n].detach().requires_grad_(case["train"]) for n in names]
            wanted = leaves + [st[n].requires_grad_(case["train"]) for n in shared]
            with torch.set_grad_enabled(case["train"]):
                u, y = sample(*leaves, *([] if case["mod"] else [None, None]))
            rows["out"].append(u.detach())
            rows["y"].append(y.detach())
            if case["train"]:
                got = torch.autograd.grad((u, y), wanted, (st["dout"][i, lo:lo + step], st["dy"][i, lo:lo + step]))
                for n, t in zip(names + shared, got):
                    if n in rows:
                        rows[n].append(t)
                    else:
                        sums[n] = sums.get(n, 0) + t
        for n, parts in rows.items():
            if parts:
                out.setdefault(n if n in ("out", "y") else "d" + n, []).append(torch.cat(parts))
        for n, t in sums.items():
            if n in shared:
                out["d" + n] = out.get("d" + n, 0) + t
            else:
                out.setdefault("d" + n, []).append(t)
    return {n: torch.stack(t) if isinstance(t, list) else t for n, t in out.items()}
