"""Layer norm and its gradients on the GPU against 64-bit definitions, with the bounds of block_util."""
import pytest
import torch

from block_util import DTYPES, E, U32, directional, out_u, randn, within

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def inputs_of(rows, d, dtype, seed=0):
    x = randn((rows, d), torch.float32, seed, 2.0) + randn((d,), torch.float32, seed + 1, 1.0, 0.5)
    return x.to(dtype), randn((d,), dtype, seed + 2, 0.2, 1.0), randn((d,), dtype, seed + 3, 0.2), randn((rows, d), dtype, seed + 4)


def run(rl, x, gamma, beta, dy, eps=EPS, sums=True):
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(x.shape[:-1], dtype=torch.float32, device="cuda") for _ in range(2))
    dg, db = (torch.full((x.shape[-1],), float("nan"), device="cuda") for _ in range(2)) if sums else (None, None)
    rl.layer_norm(x, gamma, beta, eps, y, mean, rstd)
    rl.layer_norm_backward(x, gamma, mean, rstd, dy, dx, dg, db, rl.layer_norm_backward_workspace(x))
    torch.cuda.synchronize()
    return y, mean, rstd, dx, dg, db


def check(x, gamma, beta, dy, got, eps=EPS):
    y, mean, rstd, dx, dg, db = got
    rows, d = x.shape
    u, n = out_u(x.dtype), d + 8                     # fp32 operations in a row's sums
    X, DY = x.double(), dy.double()
    G = torch.ones(d, dtype=torch.float64, device="cuda") if gamma is None else gamma.double()
    B = torch.zeros_like(G) if beta is None else beta.double()
    mu = X.mean(1, keepdim=True)
    var = ((X - mu) ** 2).mean(1, keepdim=True)
    rs = 1 / (var + eps).sqrt()
    xh = (X - mu) * rs
    dmu = n * U32 * X.abs().mean(1, keepdim=True)    # error of the mean, and what it does to xh
    exh = rs * dmu + (n * U32 + E) * (xh.abs() + rs * dmu) + U32 * rs * (X.abs() + mu.abs())
    within("mean", mean, mu[:, 0], (dmu + U32 * mu.abs())[:, 0])
    within("rstd", rstd, rs[:, 0], (rs * (n * U32 + E) + rs * (rs * dmu) ** 2 + rs ** 2 * dmu)[:, 0])
    ref = xh * G + B
    within("y", y, ref, u * ref.abs() + exh * G.abs() + E * (xh * G).abs() + E * B.abs())
    a = DY * G
    m1, m2 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    ref = rs * (a - m1 - xh * m2)
    mag = rs * (a.abs() + a.abs().mean(1, keepdim=True) + xh.abs() * (a * xh).abs().mean(1, keepdim=True))
    slack = rs * (exh * (a * xh).abs().mean(1, keepdim=True) + xh.abs() * (a.abs() * exh).mean(1, keepdim=True))
    within("dx", dx, ref, u * ref.abs() + (n * U32 + 2 * E) * mag + slack * 2)
    if dg is not None:
        k = rows + 16
        within("dgamma", dg, (DY * xh).sum(0), k * U32 * (DY * xh).abs().sum(0) + (DY.abs() * exh).sum(0) * 2)
        within("dbeta", db, DY.sum(0), k * U32 * DY.abs().sum(0))


# widths: one element, odd, just around a warp's and a CTA's pieces, the model widths, past the registers
SHAPES = [(1, 1), (3, 2), (5, 7), (2, 8), (33, 64), (7, 255), (9, 256), (130, 777), (1, 1536), (611, 1536), (4, 1544),
          (3, 4999), (1, 5120), (77, 5120), (5, 5128), (2, 10241), (3, 20480), (2, 33000), (2, 90000), (2500, 96)]


@pytest.mark.parametrize("rows,d", SHAPES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_against_64_bits(rl, rows, d, dname):
    x, gamma, beta, dy = inputs_of(rows, d, DTYPES[dname], seed=rows * 7 + d)
    check(x, gamma, beta, dy, run(rl, x, gamma, beta, dy))


@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_without_affine_and_without_sums(rl, dname):
    x, gamma, _, dy = inputs_of(21, 192, DTYPES[dname])
    check(x, None, None, dy, run(rl, x, None, None, dy))
    check(x, gamma, None, dy, run(rl, x, gamma, None, dy, sums=False))


@pytest.mark.parametrize("d", [64, 77, 40000])
def test_unaligned_pointers_and_outputs_in_place(rl, d):
    """Tensors that start one element past a 16-byte boundary; y written over x, dx over dy."""
    for dt in DTYPES.values():
        x, gamma, beta, dy = inputs_of(11, d, dt)
        off = lambda t: torch.cat([t.new_zeros(1), t.flatten()])[1:].view(t.shape)  # noqa: E731
        check(x, gamma, beta, dy, run(rl, off(x), off(gamma), off(beta), off(dy)))
        y, mean, rstd, dx, dg, db = run(rl, x, gamma, beta, dy)
        x2, dy2 = x.clone(), dy.clone()
        rl.layer_norm_backward(x, gamma, mean, rstd, dy2, dy2, dg, db, rl.layer_norm_backward_workspace(x))
        rl.layer_norm(x2, gamma, beta, EPS, x2)
        torch.cuda.synchronize()
        assert torch.equal(x2, y) and torch.equal(dy2, dx)


def test_constant_rows_and_large_offsets(rl):
    """A constant row has variance 0: y = beta, rstd = eps^-1/2.  An offset of 4096 leaves the centred row exact."""
    x = torch.full((4, 512), 3.0, device="cuda")
    x[2] += 4096.0
    x[3] = torch.where(torch.arange(512, device="cuda") % 2 == 0, 4097.0, 4095.0)
    gamma, beta = randn((512,), torch.float32, 1), randn((512,), torch.float32, 2)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    rl.layer_norm(x, gamma, beta, EPS, y, mean, rstd)
    for r in range(3):
        assert torch.equal(y[r], beta) and abs(rstd[r].item() * EPS ** 0.5 - 1) < 1e-6
    sign = torch.where(torch.arange(512, device="cuda") % 2 == 0, 1.0, -1.0)
    within("y", y[3], (sign * gamma + beta).double(), 2e-6 * (gamma.abs() + beta.abs()).double())


def test_same_bits_and_streams(rl):
    """Two calls give the same bits; a side stream orders the call after the work it waits for."""
    x, gamma, beta, dy = inputs_of(3001, 1536, torch.bfloat16)
    a, b = run(rl, x, gamma, beta, dy), run(rl, x, gamma, beta, dy)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    side, y = torch.cuda.Stream(), torch.zeros_like(x)
    with torch.cuda.stream(side):
        z = x * 1.0
        rl.layer_norm(z, gamma, beta, EPS, y)
    side.synchronize()
    assert torch.equal(y, a[0])


def test_gradient_against_differences(rl):
    x, gamma, beta, dy = inputs_of(17, 200, torch.float32)
    _, _, _, dx, dg, db = run(rl, x, gamma, beta, dy)

    def loss(x_, g_, b_):
        y = torch.empty_like(x_)
        rl.layer_norm(x_, g_, b_, EPS, y)
        return (y.double() * dy.double()).sum().item()
    args, scale = [x, gamma, beta], dy.double().norm().item() * 60.0      # |y| about 60
    for i, grad in enumerate((dx, dg, db)):
        d = torch.sign(randn(args[i].shape, torch.float32, 9 + i))
        f = lambda t: loss(*[t if j == i else args[j] for j in range(3)])  # noqa: E731
        want, gap = directional(f, args[i], d)
        # an fp32 forward is within 2^-20 of its value at either end of the step
        assert abs((grad.double() * d.double()).sum().item() - want) <= gap + 2 * scale * 2.0 ** -20 * 2 ** 6


def test_autograd_function(rl):
    x, gamma, beta, dy = inputs_of(40, 320, torch.float32)
    x, dy = x.view(5, 8, 320), dy.view(5, 8, 320)
    leaves = [t.clone().requires_grad_() for t in (x, gamma, beta)]
    ref = [t.double().clone().requires_grad_() for t in (x, gamma, beta)]
    rl.LayerNormFunction.apply(*leaves, EPS).backward(dy)
    torch.nn.functional.layer_norm(ref[0], (320,), ref[1], ref[2], EPS).backward(dy.double())
    for a, b in zip(leaves, ref):
        assert (a.grad.double() - b.grad).norm() <= 1e-5 * b.grad.norm()


def test_refusals(rl):
    x = torch.zeros((4, 64), device="cuda")
    y, m = torch.empty_like(x), torch.empty(4, device="cuda")
    with pytest.raises(ValueError):
        rl.layer_norm(x.half(), None, None, EPS, y)
    with pytest.raises(ValueError):
        rl.layer_norm(x.t(), None, None, EPS, torch.empty_like(x.t().contiguous()))
    with pytest.raises(ValueError):
        rl.layer_norm(x, torch.ones(63, device="cuda"), None, EPS, y)
    with pytest.raises(ValueError):
        rl.layer_norm(x, None, None, EPS, y.bfloat16())
    for bad in (dict(mean=m), dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(rl.RolaError):
            rl.layer_norm(x, None, None, bad.get("eps", EPS), y, bad.get("mean"))
    with pytest.raises(rl.RolaError):
        rl.layer_norm_backward(x, None, m, m, x, y, torch.empty(64, device="cuda"), torch.empty(64, device="cuda"),
                               torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(rl.RolaError):
        rl.layer_norm(x[:0], None, None, EPS, y[:0])
