"""Linear layers with their epilogue, and their gradients, on the GPU against 64-bit definitions, with the bounds of block_util."""
import pytest
import torch

from block_util import DTYPES, E, U16, U32, directional, out_u, randn, within

pytestmark = pytest.mark.gpu
ACTS = ["identity", "silu", "tanh", "relu", "gelu"]


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def nan(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


class Case:
    def __init__(self, rl, m, k, n, act, dtype, bias=True, residual=True, seed=0):
        self.rl, self.act, self.dtype, self.m, self.k, self.n = rl, act, dtype, m, k, n
        self.c = rl.make_linear_config(m, k, n, act, rl.ROLA_BF16 if dtype == torch.bfloat16 else rl.ROLA_FP32)
        self.X, self.W = randn((m, k), dtype, seed), randn((n, k), dtype, seed + 1, k ** -0.5)
        self.b = randn((n,), dtype, seed + 2, 0.3) if bias else None
        self.R = randn((m, n), dtype, seed + 3) if residual else None
        self.dY = randn((m, n), dtype, seed + 4)

    def forward(self):
        rl, c = self.rl, self.c
        Y, ws = nan(self.m, self.n, dtype=self.dtype), rl.linear_workspace(c)
        rl.linear(c, self.X, self.W, self.b, self.R, Y, ws)
        assert rl.get_device_status(ws) == rl.ROLA_OK
        return Y

    def run(self):
        rl, c = self.rl, self.c
        Y, Z = nan(self.m, self.n, dtype=self.dtype), nan(self.m, self.n)
        ws, bws = rl.linear_workspace(c), rl.linear_backward_workspace(c)
        bws.fill_(0xFF)                                      # NaN wherever a sum would read what it has not written
        dX, dW, db = nan(self.m, self.k, dtype=self.dtype), nan(self.n, self.k, dtype=self.dtype), nan(self.n)
        rl.linear_train(c, self.X, self.W, self.b, self.R, Y, Z, ws)
        rl.linear_backward(c, self.X, self.W, Z, self.dY, dX, dW, db, bws)
        assert rl.get_device_status(ws) == rl.ROLA_OK and rl.get_device_status(bws) == rl.ROLA_OK
        return dict(Y=Y, Z=Z, dX=dX, dW=dW, db=db)

    def check(self, got):
        """First-order bounds; phi' <= 1.13 and |phi''| <= 0.8 for every map here."""
        u = out_u(self.dtype)
        r = U16 if self.dtype == torch.bfloat16 else 0.0     # dZ as an operand of the products (the identity's is dY itself)
        x, w, dy = self.X.double(), self.W.double(), self.dY.double()
        z, ez = x @ w.t(), (self.k * U32 + E) * (x.abs() @ w.abs().t())
        if self.b is not None:
            z, ez = z + self.b.double(), ez + E * self.b.double().abs()
        a, da = phi(self.act, z)
        ea = 1.13 * ez + E * (a.abs() + ez) if self.act != "identity" else ez
        y = a if self.R is None else a + self.R.double()
        within("Y", got["Y"], y, (ea + U32 * y.abs()) * (1 + u) + u * y.abs())
        if "dX" not in got:
            return
        within("Z", got["Z"], z, ez)
        dz = dy * da
        eda = torch.zeros_like(z) if self.act == "identity" else 0.8 * ez + E
        if self.act == "relu":
            eda = torch.where(z.abs() <= ez, 1.0, E)         # within rounding of the kink phi' is 0 or 1
        edz = dy.abs() * eda + E * dz.abs()
        within("db", got["db"], dz.sum(0), edz.sum(0) + (self.m * U32 + E) * dz.abs().sum(0))
        if self.act != "identity":
            edz = edz * (1 + r) + r * dz.abs()
        else:
            edz = torch.zeros_like(z)
        for name, A, eA, B in (("dX", dz, edz, w), ("dW", dz.t(), edz.t(), x)):
            ref, size = A @ B, A.abs() @ B.abs()
            within(name, got[name], ref, (eA @ B.abs() + (A.shape[1] * U32 + E) * size) * (1 + u) + u * ref.abs())


def phi(act, z):
    if act == "identity":
        return z, torch.ones_like(z)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if act == "tanh":
        return torch.tanh(z), 1 - torch.tanh(z) ** 2
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    cdf = torch.special.ndtr(z)
    return z * cdf, cdf + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5


# (tokens, d_in, d_out): the smallest widths, partial tiles in every direction, whole tiles, one token and few
SIZES = [(1, 8, 8), (3, 16, 8), (2, 8, 4104), (1, 1536, 4096), (2, 128, 512), (9, 264, 520), (17, 72, 1032), (64, 128, 128),
         (77, 136, 264), (100, 1032, 72), (127, 64, 64), (128, 256, 256), (129, 384, 640), (256, 512, 512), (257, 72, 264),
         (333, 200, 328), (515, 512, 1288), (1100, 328, 200), (5000, 64, 136), (700, 2056, 40)]


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("act", ["identity", "gelu"])
def test_against_64_bits(rl, m, k, n, dname, act):
    case = Case(rl, m, k, n, act, DTYPES[dname], seed=m + k + n)
    got = case.run()
    case.check(got)
    assert torch.equal(case.forward(), got["Y"]), "the training forward gives other bits"


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("m", [5, 150])
def test_every_epilogue(rl, act, dname, bias, residual, m):
    case = Case(rl, m, 136, 200, act, DTYPES[dname], bias, residual, seed=50)
    case.check(case.run())


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 65, 96, 97, 130, 191, 200, 300, 400, 600, 700])
@pytest.mark.parametrize("k,n", [(1544, 2056), (64, 8200), (4104, 136)])
def test_every_token_count_where_the_form_changes(rl, m, k, n):
    case = Case(rl, m, k, n, "silu", torch.bfloat16, seed=m)
    case.check(dict(Y=case.forward()))
    case.check(case.run())


@pytest.mark.parametrize("m,k,n,act", [(9000, 520, 264, "identity"), (33000, 72, 72, "silu"), (20000, 1544, 136, "identity"), (6001, 264, 2056, "tanh"),
                                       (3000, 1032, 3080, "gelu")])
def test_many_tokens(rl, m, k, n, act):
    """Several turns of tiles, and weights' gradients whose few tiles have a long axis of tokens."""
    case = Case(rl, m, k, n, act, torch.bfloat16, seed=m)
    case.check(case.run())


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("m", [3, 40, 300])
def test_in_place_of_the_residual(rl, dname, m):
    case = Case(rl, m, 520, 264, "gelu", DTYPES[dname])
    want, ws = case.forward(), rl.linear_workspace(case.c)
    rl.linear(case.c, case.X, case.W, case.b, case.R, case.R, ws)
    assert torch.equal(case.R, want)


@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("act", ["identity", "silu"])
@pytest.mark.parametrize("m", [7, 300])
def test_each_gradient_alone(rl, dname, act, m):
    """Those that are not wanted change nothing in the others."""
    case = Case(rl, m, 264, 520, act, DTYPES[dname])
    want, ws = case.run(), rl.linear_backward_workspace(case.c)
    Z = None if act == "identity" else want["Z"]
    for keep in (("dX",), ("dW",), ("db",), ("dX", "db"), ("dW", "db")):
        out = {n: torch.full_like(want[n], float("nan")) if n in keep else None for n in ("dX", "dW", "db")}
        rl.linear_backward(case.c, case.X, case.W, Z, case.dY, out["dX"], out["dW"], out["db"], ws)
        assert rl.get_device_status(ws) == rl.ROLA_OK
        for n in keep:
            assert torch.equal(out[n], want[n]), n


def test_large_sums_stay_finite(rl):
    """Sums of +-300: phi's exponential over- and underflows, the results do not."""
    for dt in DTYPES.values():
        for m in (40, 200):
            case = Case(rl, m, 64, 128, "identity", dt, seed=3)
            case.W = (case.W.float() * 300).to(dt)
            for act in ("silu", "gelu", "tanh"):
                case.c.act = rl.LOWRANK_ACTS[act]
                assert all(torch.isfinite(t).all() for t in case.run().values())


@pytest.mark.parametrize("m", [5, 300])
def test_what_is_not_a_number_stays_in_its_row(rl, m):
    for dt in DTYPES.values():
        case = Case(rl, m, 264, 520, "relu", dt)
        clean = case.forward()
        case.X[2, 100] = float("nan")
        got = case.forward()
        others = torch.arange(m, device="cuda") != 2
        assert torch.equal(got[others], clean[others]) and torch.isnan(got[2]).all()


@pytest.mark.parametrize("m", [1, 20, 700])
def test_same_bits_and_streams(rl, m):
    case = Case(rl, m, 520, 1032, "silu", torch.bfloat16)
    a, b = case.run(), case.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = case.run()
    side.synchronize()
    for n in a:
        assert torch.equal(a[n], b[n]) and torch.equal(a[n], c[n]), n


@pytest.mark.parametrize("m", [2, 300])
def test_captured_and_replayed(rl, m):
    case = Case(rl, m, 264, 520, "gelu", torch.bfloat16)
    want, c = case.run(), case.c
    ws, bws = rl.linear_workspace(c), rl.linear_backward_workspace(c)
    got = {n: torch.full_like(t, float("nan")) for n, t in want.items()}

    def step():
        rl.linear_train(c, case.X, case.W, case.b, case.R, got["Y"], got["Z"], ws)
        rl.linear_backward(c, case.X, case.W, got["Z"], case.dY, got["dX"], got["dW"], got["db"], bws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t in got.values():
        t.fill_(float("nan"))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(got[n], want[n]), n
    case.X.neg_()                                            # new inputs in the same buffers
    graph.replay()
    again = case.run()
    for n in again:
        assert torch.equal(got[n], again[n]), n


@pytest.mark.parametrize("m", [12, 200])
def test_gradient_against_differences(rl, m):
    case = Case(rl, m, 64, 96, "gelu", torch.float32, seed=7)
    got = case.run()
    scale = case.dY.double().norm().item() * got["Y"].double().norm().item()
    for i, (name, grad) in enumerate((("X", got["dX"]), ("W", got["dW"]), ("b", got["db"]), ("R", case.dY))):
        t = getattr(case, name)
        d = torch.sign(randn(t.shape, torch.float32, 9 + i)) * (0.1 if name == "W" else 1.0)

        def f(v):
            setattr(case, name, v)
            return (case.forward().double() * case.dY.double()).sum().item()
        want, gap = directional(f, t, d)
        setattr(case, name, t)
        assert abs((grad.double() * d.double()).sum().item() - want) <= gap + 2 * scale * 2.0 ** -20 * 2 ** 6, name


@pytest.mark.parametrize("act,bias,residual", [("silu", True, True), ("identity", True, False), ("gelu", False, True)])
def test_autograd_function(rl, act, bias, residual):
    case = Case(rl, 24, 64, 128, act, torch.float32, bias, residual)
    lead = (2, 12)
    a = [None if t is None else t.clone().requires_grad_() for t in (case.X.view(*lead, 64), case.W, case.b, None if case.R is None else case.R.view(*lead, 128))]
    b = [None if t is None else t.detach().double().requires_grad_() for t in a]
    rl.LinearFunction.apply(*a, act).backward(case.dY.view(*lead, 128))
    z = torch.nn.functional.linear(b[0], b[1], b[2])
    y = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "identity": lambda t: t}[act](z)
    (y if b[3] is None else y + b[3]).backward(case.dY.double().view(*lead, 128))
    for s, t in zip(a, b):
        assert s is None or (s.grad.double() - t.grad).norm() <= 1e-5 * t.grad.norm()


def test_autograd_of_some_inputs(rl):
    case = Case(rl, 10, 64, 128, "silu", torch.float32)
    ref = case.X.double().requires_grad_(), case.W.double().requires_grad_(), case.b.double().requires_grad_()
    torch.nn.functional.silu(torch.nn.functional.linear(*ref)).backward(case.dY.double())
    for i in range(3):
        leaves = [t.clone().requires_grad_(i == j) for j, t in enumerate((case.X, case.W, case.b))]
        rl.LinearFunction.apply(*leaves, None, "silu").backward(case.dY)
        for j, t in enumerate(leaves):
            assert (t.grad is None) == (i != j)
        assert (leaves[i].grad.double() - ref[i].grad).norm() <= 1e-5 * ref[i].grad.norm()


def test_a_residual_of_another_shape_gets_its_gradient_in_it(rl):
    case = Case(rl, 24, 64, 128, "silu", torch.float32)
    X, R = case.X.view(2, 12, 64), case.R.clone().requires_grad_()
    rl.LinearFunction.apply(X, case.W, case.b, R, "silu").backward(case.dY.view(2, 12, 128))
    assert torch.equal(R.grad, case.dY)


def test_refusals(rl):
    case = Case(rl, 4, 64, 128, "silu", torch.bfloat16)
    c, X, W, b, R = case.c, case.X, case.W, case.b, case.R
    ws, bws, Y = rl.linear_workspace(c), rl.linear_backward_workspace(c), torch.empty_like(R)
    with pytest.raises(ValueError):
        rl.linear(c, X.float(), W, b, R, Y, ws)
    with pytest.raises(ValueError):
        rl.linear(c, X, W.t().contiguous(), b, R, Y, ws)
    with pytest.raises(ValueError):
        rl.linear(c, X, W, b.float(), R, Y, ws)
    with pytest.raises(ValueError):
        rl.linear(c, X, W, b, X, Y, ws)
    with pytest.raises(ValueError):
        rl.linear(c, X, W.t().contiguous().t(), b, R, Y, ws)
    with pytest.raises(rl.RolaError):
        rl.linear(c, X, W, b, R, Y, ws[:128])
    with pytest.raises(rl.RolaError):
        rl.linear_train(c, X, W, b, R, Y, None, ws)
    Z = nan(4, 128)
    with pytest.raises(rl.RolaError):
        rl.linear_backward(c, X, W, None, R, torch.empty_like(X), None, None, bws)
    with pytest.raises(rl.RolaError):
        rl.linear_backward(c, X, W, Z, R, None, None, None, bws)
    with pytest.raises(rl.RolaError):
        rl.linear_backward(c, X, W, Z, R, torch.empty_like(X), None, None, bws[:256])
    for bad in ((0, 64, 128), (4, 60, 128), (4, 64, 4)):
        with pytest.raises(rl.RolaError):
            rl.linear_workspace(rl.make_linear_config(*bad))
