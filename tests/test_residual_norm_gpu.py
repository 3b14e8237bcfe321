"""The gated residual sum and its norms on the GPU against 64-bit definitions, with the bounds of block_util."""
import itertools

import pytest
import torch

from block_util import DTYPES, E, U32, directional, out_u, randn, within

pytestmark = pytest.mark.gpu
EPS = 1e-6
VECTORS = ("gate", "gamma_h", "gamma", "beta", "scale", "shift")


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


class Case:
    """Inputs of one call; vectors: the names of those that are there."""

    def __init__(self, rl, B, n, d, norm, branch, vectors, dtype, h=True, out_used=True, seed=0, apart=0, shift=0.0):
        self.rl, self.dtype, self.norm, self.branch = rl, dtype, norm, branch
        self.c = rl.make_residual_norm_config(B, n, d, norm, branch, EPS, apart, rl.ROLA_BF16 if dtype == torch.bfloat16 else rl.ROLA_FP32)
        self.x = randn((B, n, d), dtype, seed, 1.5, 0.3 + shift)
        self.h = randn((B, n, d), dtype, seed + 1) if h else None
        self.v = dict.fromkeys(VECTORS)
        for i, name in enumerate(vectors):
            if name in ("gate", "scale", "shift"):
                self.v[name] = randn((B, apart or d), dtype, seed + 2 + i, 0.5)[:, :d]
            else:
                self.v[name] = randn((d,), dtype, seed + 2 + i, 0.2, 0.0 if name == "beta" else 1.0)
        self.dout = randn((B, n, d), dtype, seed + 9) if out_used and h else None
        self.dy = randn((B, n, d), dtype, seed + 10) if norm != "none" else None

    def blank(self, *shape, dtype=torch.float32):
        return torch.full(shape, float("nan"), dtype=dtype, device="cuda")

    def run(self, stream=None):
        rl, c, v = self.rl, self.c, self.v
        shape = self.x.shape
        out = self.blank(*shape, dtype=self.dtype) if self.h is not None else None
        y = self.blank(*shape, dtype=self.dtype) if self.norm != "none" else None
        stats = self.blank(*shape[:2], 4)
        rl.residual_norm(c, self.x, self.h, out, y, **v, stats=stats, stream=stream)
        dx, dh = self.blank(*shape, dtype=self.dtype), None if self.h is None else self.blank(*shape, dtype=self.dtype)
        grads = {"d" + n: None if v[n] is None else self.blank(*v[n].shape) for n in VECTORS}
        ws = rl.residual_norm_backward_workspace(c)
        ws.fill_(0xFF)                                       # NaN wherever a sum would read what it has not written
        rl.residual_norm_backward(c, self.x, self.h, stats, self.dout, self.dy, dx, dh, ws, **{n: v[n] for n in VECTORS if n != "shift"},
                                  **grads, stream=stream)
        return dict(out=out, y=y, stats=stats, dx=dx, dh=dh, **grads)

    def check(self, got):
        """First-order bounds.  A row's mean of n values is within n 2^-24 of theirs; the deviation of a normalised value is at
        most that of the value, of the mean and of the size, relative to the size."""
        d = self.x.shape[-1]
        u, n32 = out_u(self.dtype), d * U32 + E
        x, dy, dout = (None if t is None else t.double() for t in (self.x, self.dy, self.dout))
        v = {n: None if t is None else t.double() for n, t in self.v.items()}
        per = lambda t: t[:, None] if t.dim() == 2 else t  # noqa: E731
        one, zero = torch.ones((), device="cuda", dtype=torch.float64), torch.zeros((), device="cuda", dtype=torch.float64)

        def normal(kind, t, et):
            """The normalised rows, 1 / size and the bound of the first, of rows known within et."""
            c = t - t.mean(-1, keepdim=True) if kind == "layer" else t
            r = 1 / (c.square().mean(-1, keepdim=True) + EPS).sqrt()
            ec = et + (et.mean(-1, keepdim=True) + n32 * t.abs().mean(-1, keepdim=True) if kind == "layer" else 0)
            vh = c * r
            # relative error of r: that of the mean square, half of it
            er = (c.abs() * ec).mean(-1, keepdim=True) * r * r + n32
            return vh, r, ec * r + vh.abs() * (er + E)

        g = per(v["gate"]) if v["gate"] is not None else one
        gh = v["gamma_h"] if v["gamma_h"] is not None else one
        if self.h is None:
            U, eU, hh, ehh, rh = x, zero * x, None, None, None
        else:
            h = self.h.double()
            hh, rh, ehh = (h, one, zero * h) if self.branch == "none" else normal(self.branch, h, zero * h)
            gg = g * gh
            U = x + gg * hh
            eU = gg.abs() * ehh + E * (gg * hh).abs() + 2 * U32 * U.abs()
            within("out", got["out"], U, eU * (1 + u) + u * U.abs())
        if self.norm != "none":
            s1 = 1 + per(v["scale"]) if v["scale"] is not None else one
            gam, bet = (v[n] if v[n] is not None else t for n, t in (("gamma", one), ("beta", zero)))
            sh = per(v["shift"]) if v["shift"] is not None else zero
            V, r, eV = normal(self.norm, U, eU)
            Y = (V * gam + bet) * s1 + sh
            size = (V * gam * s1).abs() + (bet * s1).abs() + sh.abs()
            within("y", got["y"], Y, (eV * (gam * s1).abs() + E * size) * (1 + u) + u * Y.abs())
            a = dy * gam * s1
            m = (a * V).mean(-1, keepdim=True)
            em = (a.abs() * eV).mean(-1, keepdim=True) + n32 * (a * V).abs().mean(-1, keepdim=True)
            core = a - V * m
            ecore = E * a.abs() + V.abs() * em + eV * m.abs() + E * (V * m).abs()
            if self.norm == "layer":
                core = core - a.mean(-1, keepdim=True)
                ecore = ecore + n32 * a.abs().mean(-1, keepdim=True)
            rel = (eV.square().mean(-1, keepdim=True)).sqrt() + n32 + E      # of r, by the size of the normalised rows' error
            t, et = r * core, r * ecore + (r * core).abs() * rel
        else:
            t, et = zero * x, zero * x
        if dout is not None:
            t, et = t + dout, et + E * dout.abs()
        et = et + E * t.abs()
        within("dx", got["dx"], t, et * (1 + u) + u * t.abs())
        if self.h is not None:
            e, ee = t * gg, et * gg.abs() + E * (t * gg).abs()
            if self.branch != "none":
                m = (e * hh).mean(-1, keepdim=True)
                em = (ee * hh.abs() + e.abs() * ehh).mean(-1, keepdim=True) + n32 * (e * hh).abs().mean(-1, keepdim=True)
                core, ecore = e - hh * m, ee + hh.abs() * em + ehh * m.abs() + E * (hh * m).abs()
                if self.branch == "layer":
                    core, ecore = core - e.mean(-1, keepdim=True), ecore + ee.mean(-1, keepdim=True) + n32 * e.abs().mean(-1, keepdim=True)
                rel = (ehh.square().mean(-1, keepdim=True)).sqrt() + n32 + E
                e, ee = rh * core, rh * ecore + (rh * core).abs() * rel
            within("dh", got["dh"], e, ee * (1 + u) + (u + E) * e.abs())
        rows = self.x.shape[1]

        def column(name, terms, eterms, dims, n):
            if got[name] is not None:
                within(name, got[name], terms.sum(dims), eterms.sum(dims) + (n * U32 + 4 * E) * terms.abs().sum(dims))
        per_sample, all_rows = (1, rows), ((0, 1), rows * self.x.shape[0])
        if self.h is not None:
            et_hh = et * hh.abs() + t.abs() * ehh
            column("dgate", t * hh * gh, et_hh * gh.abs(), *per_sample)
            column("dgamma_h", t * hh * g, et_hh * g.abs(), *all_rows)
        if self.norm != "none":
            eA = dy.abs() * eV
            column("dscale", dy * (V * gam + bet), eA * gam.abs() + E * (dy.abs() * (V * gam).abs() + (dy * bet).abs()), *per_sample)
            column("dshift", dy, zero * dy, *per_sample)
            column("dgamma", dy * V * s1, eA * s1.abs(), *all_rows)
            column("dbeta", dy * s1, zero * dy, *all_rows)


ALL = VECTORS
SOME = [("gate", "scale", "shift"), ("gamma", "beta"), (), ("gate", "gamma", "scale")]
# (groups, rows, d): one row, one element, widths of a warp and of a CTA with ragged and whole pieces, rows of no vector load,
# samples of one row, a width past the registers
SIZES = [(1, 1, 1), (1, 1, 5120), (2, 1, 8), (1, 3, 64), (3, 5, 7), (2, 33, 256), (5, 9, 264), (1, 130, 520), (2, 70, 1536), (4, 3, 777),
         (1, 37, 2051), (3, 11, 2560), (2, 5, 5120), (1, 9, 4104), (2, 3, 8200), (1, 5, 9001), (40, 1, 136), (70, 2, 24), (1, 2, 20488)]


@pytest.mark.parametrize("B,n,d", SIZES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("norm,branch", [("layer", "none"), ("rms", "rms"), ("layer", "layer")])
def test_against_64_bits(rl, B, n, d, dname, norm, branch):
    case = Case(rl, B, n, d, norm, branch, [v for v in ALL if branch != "none" or v != "gamma_h"], DTYPES[dname], seed=B + n + d)
    case.check(case.run())


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("d", [96, 520, 1536, 333])
@pytest.mark.parametrize("norm,branch,h", [("layer", "none", True), ("rms", "layer", True), ("rms", "none", False), ("layer", "none", False),
                                           ("none", "none", True), ("none", "rms", True)])
def test_every_form_with_some_of_the_vectors(rl, d, dname, norm, branch, h):
    for vectors, out_used in itertools.product(SOME, (True, False)):
        names = [v for v in vectors if (h or v != "gate") and (norm != "none" or v == "gate")]
        if branch != "none" and len(vectors) % 2:
            names.append("gamma_h")
        if norm == "none" and not out_used:
            continue
        case = Case(rl, 2, 19, d, norm, branch, names, DTYPES[dname], h=h, out_used=out_used, seed=d)
        case.check(case.run())


@pytest.mark.parametrize("d,apart", [(256, 1536), (1536, 1537), (777, 4662), (5120, 30720)])
@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_vectors_that_are_slices_of_a_modulation(rl, d, apart, dname):
    case = Case(rl, 3, 8, d, "layer", "none", ("gate", "scale", "shift"), DTYPES[dname], apart=apart)
    case.check(case.run())


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("d", [777, 1286, 1537, 2059, 3583, 5119, 8191])
def test_many_rows_of_small_pieces(rl, d, dname):
    """Widths of no 16-byte pieces, one for each number of threads, over several turns of the ring."""
    case = Case(rl, 5, 521 if d < 4000 else 131, d, "layer", "rms", ALL, DTYPES[dname], seed=d)
    case.check(case.run())


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("d", [777, 1536])
@pytest.mark.parametrize("rows", [456, 457, 1216, 1217])
def test_where_few_rows_end(rl, rows, d, dname):
    case = Case(rl, 1, rows, d, "rms", "layer", ALL, DTYPES[dname], seed=rows)
    case.check(case.run())


@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_many_rows_per_cta(rl, dname):
    """Samples that begin and end within a CTA's rows, over several turns of its ring."""
    for B, n, d in ((3, 4001, 264), (1, 9001, 1536), (700, 13, 520), (2, 3000, 5120)):
        case = Case(rl, B, n, d, "layer", "rms", ALL, DTYPES[dname], seed=n)
        case.check(case.run())


@pytest.mark.parametrize("d", [64, 1536, 777, 9000])
def test_in_place(rl, d):
    """out and y in place of x and h, dx and dh in place of dout and dy: the same bits."""
    for dt in DTYPES.values():
        case = Case(rl, 2, 50, d, "layer", "rms", ALL, dt)
        want = case.run()
        for swap in (False, True):
            x, h, dout, dy = (t.clone() for t in (case.x, case.h, case.dout, case.dy))
            out, y = (h, x) if swap else (x, h)
            rl.residual_norm(case.c, x, h, out, y, **case.v)
            assert torch.equal(out, want["out"]) and torch.equal(y, want["y"])
            dx, dh = (dy, dout) if swap else (dout, dy)
            v = {k: t for k, t in case.v.items() if k != "shift"}
            dgate = torch.empty_like(want["dgate"])
            rl.residual_norm_backward(case.c, case.x, case.h, want["stats"], dout, dy, dx, dh, rl.residual_norm_backward_workspace(case.c),
                                      **v, dgate=dgate)
            assert torch.equal(dx, want["dx"]) and torch.equal(dh, want["dh"]) and torch.equal(dgate, want["dgate"])


@pytest.mark.parametrize("d", [256, 1536, 777])
def test_same_bits_and_streams(rl, d):
    case = Case(rl, 3, 400, d, "rms", "layer", ALL, torch.bfloat16)
    a, b = case.run(), case.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = case.run()
    side.synchronize()
    for n in a:
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], c[n]), n


def test_rows_of_a_large_offset_and_of_nothing(rl):
    """A common offset of 1000 sizes does not cancel in the variance; rows of one value give y = beta and finite gradients."""
    case = Case(rl, 1, 40, 1536, "layer", "none", ("gate", "gamma", "beta"), torch.float32, shift=1000.0)
    case.check(case.run())
    for d in (64, 777, 1536):
        case = Case(rl, 1, 4, d, "layer", "layer", ("gate", "gamma_h", "gamma", "beta"), torch.float32)
        case.x.fill_(3.0), case.h.fill_(-2.0)
        got = case.run()
        assert torch.equal(got["y"], case.v["beta"].expand_as(got["y"])) and torch.equal(got["out"], case.x)
        assert all(torch.isfinite(t).all() for t in got.values() if t is not None)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_a_number_stays_in_its_row(rl, bad):
    case = Case(rl, 2, 30, 520, "layer", "rms", ALL, torch.bfloat16)
    clean = case.run()
    case.x[1, 7, 100] = bad
    got = case.run()
    others = torch.ones(2, 30, dtype=torch.bool, device="cuda")
    others[1, 7] = False
    for n in ("out", "y", "dx", "dh"):
        assert torch.equal(got[n][others], clean[n][others])
    assert torch.isnan(got["y"][1, 7]).all()


def test_gradient_against_differences(rl):
    case = Case(rl, 2, 9, 48, "layer", "rms", ALL, torch.float32, seed=3)
    got = case.run()
    leaves = dict(x=case.x, h=case.h, **case.v)
    grads = dict(x=got["dx"], h=got["dh"], **{n: got["d" + n] for n in VECTORS})
    scale = case.dout.double().norm().item() * got["out"].double().norm().item() + case.dy.double().norm().item() * got["y"].double().norm().item()
    for i, name in enumerate(leaves):
        direction = torch.sign(randn(leaves[name].shape, torch.float32, 20 + i)) * 0.25

        def f(t):
            a = dict(leaves, **{name: t})
            out, y = torch.empty_like(case.x), torch.empty_like(case.x)
            rl.residual_norm(case.c, a.pop("x"), a.pop("h"), out, y, **a)
            return ((out.double() * case.dout.double()).sum() + (y.double() * case.dy.double()).sum()).item()
        want, gap = directional(f, leaves[name], direction)
        assert abs((grads[name].double() * direction.double()).sum().item() - want) <= gap + 2 * scale * 2.0 ** -20 * 2 ** 6, name


@pytest.mark.parametrize("norm,branch,h", [("layer", "none", True), ("rms", "rms", True), ("layer", "none", False), ("none", "layer", True)])
def test_autograd_function(rl, norm, branch, h):
    names = [n for n in VECTORS if (h or n not in ("gate", "gamma_h")) and (branch != "none" or n != "gamma_h")
             and (norm != "none" or n in ("gate", "gamma_h"))]
    case = Case(rl, 2, 12, 64, norm, branch, names, torch.float32, h=h)
    mod = randn((2, 3, 64), torch.float32, 30, 0.5)

    def leaves(to):
        t = {"x": case.x, "h": case.h, "mod": mod, **{n: case.v[n] for n in ("gamma_h", "gamma", "beta")}}
        return {n: None if v is None else v.to(to).clone().requires_grad_() for n, v in t.items()}

    def vectors(t):
        return {n: t["mod"][:, i] if n in names else None for i, n in enumerate(("gate", "scale", "shift"))}

    def normal(kind, t):
        if kind == "layer":
            return torch.nn.functional.layer_norm(t, t.shape[-1:], eps=EPS)
        return t * (t.square().mean(-1, keepdim=True) + EPS).rsqrt()
    a, b = leaves(torch.float32), leaves(torch.float64)
    va, vb = vectors(a), vectors(b)
    out, y = rl.ResidualNormFunction.apply(a["x"], a["h"], va["gate"], a["gamma_h"], a["gamma"], a["beta"], va["scale"], va["shift"], norm, branch, EPS)
    ref_out = b["x"]
    if h:
        w = b["h"] if branch == "none" else normal(branch, b["h"]) * b["gamma_h"]
        ref_out = ref_out + vb["gate"][:, None] * w
    total, ref = 0.0, 0.0
    if h:
        total, ref = (out * case.dout).sum(), (ref_out * case.dout.double()).sum()
    else:
        assert out is None
    if norm != "none":
        ref_y = (normal(norm, ref_out) * b["gamma"] + b["beta"]) * (1 + vb["scale"][:, None]) + vb["shift"][:, None]
        total, ref = total + (y * case.dy).sum(), ref + (ref_y * case.dy.double()).sum()
    else:
        assert y is None
    total.backward()
    ref.backward()
    for n in a:
        if b[n] is not None and b[n].grad is not None:
            assert (a[n].grad.double() - b[n].grad).norm() <= 1e-5 * b[n].grad.norm(), n


def test_autograd_with_one_result_unused(rl):
    x, h = (randn((1, 7, 96), torch.float32, i).requires_grad_() for i in (1, 2))
    for use in (0, 1):
        x.grad = h.grad = None
        got = rl.ResidualNormFunction.apply(x, h, None, None, None, None, None, None, "layer", "none", EPS)
        got[use].square().sum().backward()
        a, b = (t.detach().double().requires_grad_() for t in (x, h))
        u = a + b
        (u if use == 0 else torch.nn.functional.layer_norm(u, (96,), eps=EPS)).square().sum().backward()
        for s, t in ((x, a), (h, b)):
            assert (s.grad.double() - t.grad).norm() <= 1e-5 * t.grad.norm() + 1e-5


def test_captured_and_replayed(rl):
    case = Case(rl, 2, 40, 1536, "layer", "none", ("gate", "scale", "shift"), torch.bfloat16)
    want = case.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        case.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = case.run()
    for n, t in got.items():
        if t is not None:
            t.fill_(float("nan"))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for n in want:
        assert want[n] is None or torch.equal(got[n], want[n]), n
    first = {n: None if t is None else t.clone() for n, t in want.items()}
    case.x.neg_()                                            # new inputs in the same buffers
    graph.replay()
    again = case.run()
    assert torch.equal(got["y"], again["y"]) and torch.equal(got["dgate"], again["dgate"]) and not torch.equal(got["y"], first["y"])


def test_refusals(rl):
    case = Case(rl, 2, 5, 64, "layer", "none", ("gate", "scale"), torch.bfloat16)
    c, x, h = case.c, case.x, case.h
    out, y = torch.empty_like(x), torch.empty_like(x)
    with pytest.raises(ValueError):
        rl.residual_norm(c, x.float(), h, out, y)
    with pytest.raises(ValueError):
        rl.residual_norm(c, x, h[:, :4], out, y)
    with pytest.raises(ValueError):
        rl.residual_norm(c, x, h, out, y, gate=torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")[:, :64])
    with pytest.raises(ValueError):
        rl.residual_norm(c, x, h, out, y, gamma=torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda"))
    for bad in (dict(out=None), dict(y=None), dict(out=y), dict(h=None), dict(gamma_h=torch.zeros(64, dtype=torch.bfloat16, device="cuda"))):
        a = dict(h=h, out=out, y=y) | {k: v for k, v in bad.items() if k in ("h", "out", "y")}
        with pytest.raises(rl.RolaError):
            rl.residual_norm(c, x, a["h"], a["out"], a["y"], **{k: v for k, v in bad.items() if k not in a})
    ws, stats = rl.residual_norm_backward_workspace(c), torch.zeros((2, 5, 4), device="cuda")
    dx, dh = torch.empty_like(x), torch.empty_like(x)
    with pytest.raises(rl.RolaError):
        rl.residual_norm_backward(c, x, h, stats, x, h, dx, dh, ws[:256])
    with pytest.raises(rl.RolaError):
        rl.residual_norm_backward(c, x, h, stats, x, h, dx, dh, ws, dgate=torch.zeros(2, 64, device="cuda"))
    with pytest.raises(rl.RolaError):
        rl.residual_norm_backward(c, x, h, stats, x, h, dx, dx, ws)
    with pytest.raises(ValueError):
        rl.residual_norm_backward(c, x, h, stats, x, h, dx, dh, ws, gate=case.v["gate"], dgate=torch.zeros(64, device="cuda"))
    for bad in ((0, 5, 64), (2, 0, 64), (2, 5, 0)):
        with pytest.raises(rl.RolaError):
            rl.residual_norm_backward_workspace(rl.make_residual_norm_config(*bad))


@pytest.mark.parametrize("skip", [1, 2, 4])
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("d", [2, 30, 778, 1536, 2050])
def test_tensors_that_start_anywhere(rl, d, dname, skip):
    """Every tensor `skip` elements past a 16-byte boundary, with a guard on both sides."""
    case = Case(rl, 2, 9, d, "layer", "rms", ALL, DTYPES[dname], seed=d)
    want = case.run()
    made = []

    def moved(t, fill=None):
        buf = torch.full((t.numel() + 64,), 7.0, dtype=t.dtype, device="cuda")
        view = buf[16 + skip:16 + skip + t.numel()].view(t.shape)
        view.copy_(t if fill is None else torch.full_like(t, fill))
        made.append((buf, t.numel()))
        return view
    case.x, case.h, case.dout, case.dy = (moved(t) for t in (case.x, case.h, case.dout, case.dy))
    case.v = {n: moved(t) for n, t in case.v.items()}
    blank = {n: moved(t, float("nan")) for n, t in want.items() if n in ("out", "y", "dx", "dh")}
    stats, ws = torch.empty_like(want["stats"]), rl.residual_norm_backward_workspace(case.c)
    grads = {"d" + n: moved(want["d" + n], float("nan")) for n in VECTORS}
    rl.residual_norm(case.c, case.x, case.h, blank["out"], blank["y"], **case.v, stats=stats)
    rl.residual_norm_backward(case.c, case.x, case.h, stats, case.dout, case.dy, blank["dx"], blank["dh"], ws,
                              **{n: t for n, t in case.v.items() if n != "shift"}, **grads)
    case.check(dict(blank, stats=stats, **grads))
    for buf, n in made:
        assert (buf[:16 + skip] == 7.0).all() and (buf[16 + skip + n:] == 7.0).all()
