"""The gated feed-forward and its gradients on the GPU against 64-bit definitions, with the bounds of block_util."""
import pytest
import torch

from block_util import DTYPES, E, U16, U32, directional, out_u, randn, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def inputs_of(m, d, f, dtype, seed=0):
    return (randn((m, d), dtype, seed), randn((f, d), dtype, seed + 1, d ** -0.5), randn((f, d), dtype, seed + 2, d ** -0.5),
            randn((d, f), dtype, seed + 3, f ** -0.5), randn((m, d), dtype, seed + 4))


def nan_like(*ts):
    return [torch.full_like(t, float("nan")) for t in ts]


def run(rl, act, X, Wg, Wu, Wd, dY=None):
    c = rl.make_ffn_config(X.shape[0], X.shape[1], Wg.shape[0], act, rl.ROLA_BF16 if X.dtype == torch.bfloat16 else rl.ROLA_FP32)
    ws = rl.ffn_workspace(c)
    (Y,) = nan_like(X)
    rl.ffn(c, X, Wg, Wu, Wd, Y, ws)
    assert rl.get_device_status(ws) == rl.ROLA_OK
    if dY is None:
        return Y
    (Y2,) = nan_like(X)
    G, U = (torch.full((X.shape[0], Wg.shape[0]), float("nan"), device="cuda") for _ in range(2))
    dX, dWg, dWu, dWd = nan_like(X, Wg, Wu, Wd)
    bws = rl.ffn_backward_workspace(c)
    rl.ffn_train(c, X, Wg, Wu, Wd, Y2, G, U, ws)
    rl.ffn_backward(c, X, Wg, Wu, Wd, G, U, dY, dX, dWg, dWu, dWd, bws)
    assert rl.get_device_status(ws) == rl.ROLA_OK and rl.get_device_status(bws) == rl.ROLA_OK
    assert torch.equal(Y, Y2), "the training forward gives other bits"
    return Y, G, U, dX, dWg, dWu, dWd


def phi(act, g):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if act == "identity":
        return g, torch.ones_like(g)
    if act == "tanh":
        return torch.tanh(g), 1 - torch.tanh(g) ** 2
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    cdf = torch.special.ndtr(g)
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5


def check(act, X, Wg, Wu, Wd, got, dY=None):
    m, d = X.shape
    f = Wg.shape[0]
    u = out_u(X.dtype)
    r = U16 if X.dtype == torch.bfloat16 else 0.0        # H, dG and dU as operands of the next product
    x, wg, wu, wd = (t.double() for t in (X, Wg, Wu, Wd))
    G, U = x @ wg.t(), x @ wu.t()
    eG, eU = ((d * U32 + E) * (x.abs() @ w.abs().t()) for w in (wg, wu))
    a, da = phi(act, G)
    # |phi'| <= 1.13 and |phi''| <= 0.8 for every map here; within rounding of relu's kink phi' is 0 or 1
    ea, eda = 1.13 * eG + E * (a.abs() + eG), 0.8 * eG + E
    H = a * U
    eH = ea * U.abs() + a.abs() * eU + r * H.abs() + E * H.abs()
    Y = H @ wd.t()
    eY = eH @ wd.abs().t() + (f * U32 + E) * (H.abs() @ wd.abs().t())
    y = got if dY is None else got[0]
    within("Y", y, Y, eY * (1 + u) + u * Y.abs())
    if dY is None:
        return
    within("G", got[1], G, eG)
    within("U", got[2], U, eU)
    dy = dY.double()
    dH = dy @ wd
    edH = (d * U32 + E) * (dy.abs() @ wd.abs())
    dG, dU = dH * U * da, dH * a
    if act == "relu":
        eda = torch.where(G.abs() <= eG, 1.0, eda)
    edG = edH * (U * da).abs() + dH.abs() * (eU * da.abs() + U.abs() * eda) + (r + E) * dG.abs()
    edU = edH * a.abs() + dH.abs() * ea + (r + E) * dU.abs()
    def product(name, out, *terms):                       # terms: (A, eA, B), summed A @ B
        ref = sum(A @ B for A, _, B in terms)
        n = sum(A.shape[1] for A, _, _ in terms)
        err = sum(eA @ B.abs() + (n * U32 + E) * (A.abs() @ B.abs()) for A, eA, B in terms)
        within(name, out, ref, err * (1 + u) + u * ref.abs())
    product("dX", got[3], (dG, edG, wg), (dU, edU, wu))
    product("dW_gate", got[4], (dG.t(), edG.t(), x))
    product("dW_up", got[5], (dU.t(), edU.t(), x))
    ref = dy.t() @ H
    err = dy.abs().t() @ eH + (m * U32 + E) * (dy.abs().t() @ H.abs())
    within("dW_down", got[6], ref, err * (1 + u) + u * ref.abs())


# (tokens, d_model, d_ff): the smallest widths, partial tiles in every direction, whole tiles, one token and few
SIZES = [(1, 8, 8), (3, 16, 8), (1, 1536, 4096), (2, 128, 512), (9, 264, 520), (17, 72, 1032), (64, 128, 128), (77, 136, 264), (100, 1032, 72),
         (127, 64, 64), (128, 256, 256), (129, 384, 640), (333, 200, 328), (515, 512, 1288), (1100, 328, 200)]


@pytest.mark.parametrize("m,d,f", SIZES)
@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_against_64_bits(rl, m, d, f, dname):
    X, Wg, Wu, Wd, dY = inputs_of(m, d, f, DTYPES[dname], seed=m + d + f)
    check("silu", X, Wg, Wu, Wd, run(rl, "silu", X, Wg, Wu, Wd, dY), dY)


@pytest.mark.parametrize("act", ["identity", "tanh", "relu", "gelu"])
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("m", [5, 150])
def test_feature_maps(rl, act, dname, m):
    X, Wg, Wu, Wd, dY = inputs_of(m, 136, 200, DTYPES[dname], seed=50)
    check(act, X, Wg, Wu, Wd, run(rl, act, X, Wg, Wu, Wd, dY), dY)


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 65, 96, 130, 200])
def test_every_small_token_count_at_a_long_width(rl, m):
    """Inference over the token counts where the form of the products changes."""
    X, Wg, Wu, Wd, _ = inputs_of(m, 1544, 2056, torch.bfloat16, seed=m)
    check("silu", X, Wg, Wu, Wd, run(rl, "silu", X, Wg, Wu, Wd))


@pytest.mark.parametrize("m,d,f", [(33, 64, 128), (40, 136, 2056), (94, 328, 1032), (129, 72, 3000), (300, 1544, 64)])
def test_fp32_products_of_few_tiles_and_a_long_axis(rl, m, d, f):
    """Tiles whose K axis several CTAs share, by 2 to 8, the last rows and columns of a tile empty."""
    X, Wg, Wu, Wd, dY = inputs_of(m, d, f, torch.float32, seed=m)
    check("silu", X, Wg, Wu, Wd, run(rl, "silu", X, Wg, Wu, Wd, dY), dY)
    assert all(torch.equal(s, t) for s, t in zip(run(rl, "gelu", X, Wg, Wu, Wd, dY), run(rl, "gelu", X, Wg, Wu, Wd, dY)))


def test_large_gates_stay_finite(rl):
    """Gates of +-300: phi's exponential over- and underflows, the products do not."""
    for dt in DTYPES.values():
        X, Wg, Wu, Wd, dY = inputs_of(40, 64, 128, dt, seed=3)
        Wg = (Wg.float() * 300).to(dt)
        for act in ("silu", "gelu", "tanh"):
            for t in run(rl, act, X, Wg, Wu, Wd, dY):
                assert torch.isfinite(t).all()


@pytest.mark.parametrize("m", [1, 20, 700])
def test_same_bits_and_streams(rl, m):
    X, Wg, Wu, Wd, dY = inputs_of(m, 520, 1032, torch.bfloat16)
    a, b = run(rl, "silu", X, Wg, Wu, Wd, dY), run(rl, "silu", X, Wg, Wu, Wd, dY)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = run(rl, "silu", X * 1.0, Wg, Wu, Wd, dY)
    side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(a, c))


def test_gradient_against_differences(rl):
    args = list(inputs_of(30, 64, 96, torch.float32, seed=7))
    dY = args.pop()
    Y, _, _, *grads = run(rl, "silu", *args, dY)
    scale = dY.double().norm().item() * Y.double().norm().item()
    for i, grad in enumerate(grads):
        d = torch.sign(randn(args[i].shape, torch.float32, 9 + i)) * (1.0 if i == 0 else 0.1)
        f = lambda t: (run(rl, "silu", *[t if j == i else args[j] for j in range(4)]).double() * dY.double()).sum().item()  # noqa: E731
        want, gap = directional(f, args[i], d)
        assert abs((grad.double() * d.double()).sum().item() - want) <= gap + 2 * scale * 2.0 ** -20 * 2 ** 6


def test_autograd_function(rl):
    X, Wg, Wu, Wd, dY = inputs_of(24, 64, 128, torch.float32)
    X, dY = X.view(2, 12, 64), dY.view(2, 12, 64)
    leaves = [t.clone().requires_grad_() for t in (X, Wg, Wu, Wd)]
    ref = [t.double().clone().requires_grad_() for t in (X, Wg, Wu, Wd)]
    rl.FfnFunction.apply(*leaves, "silu").backward(dY)
    lin = torch.nn.functional.linear
    lin(torch.nn.functional.silu(lin(ref[0], ref[1])) * lin(ref[0], ref[2]), ref[3]).backward(dY.double())
    for a, b in zip(leaves, ref):
        assert (a.grad.double() - b.grad).norm() <= 1e-5 * b.grad.norm()


def test_refusals(rl):
    X, Wg, Wu, Wd, dY = inputs_of(4, 64, 128, torch.bfloat16)
    c = rl.make_ffn_config(4, 64, 128)
    ws, Y = rl.ffn_workspace(c), torch.empty_like(X)
    with pytest.raises(ValueError):
        rl.ffn(c, X.float(), Wg, Wu, Wd, Y, ws)
    with pytest.raises(ValueError):
        rl.ffn(c, X, Wg, Wu, Wg, Y, ws)
    with pytest.raises(ValueError):
        rl.ffn(c, X, Wg, Wu, Wd.t().contiguous().t(), Y, ws)
    with pytest.raises(rl.RolaError):
        rl.ffn(c, X, Wg, Wu, Wd, Y, ws[:256])
    with pytest.raises(rl.RolaError):
        rl.ffn(c, X, Wg, Wu, Wd, Y, torch.empty(ws.numel() + 16, dtype=torch.uint8, device="cuda")[16:])
    with pytest.raises(rl.RolaError):
        rl.ffn_train(c, X, Wg, Wu, Wd, Y, None, None, ws)
    for bad in ((0, 64, 128), (4, 60, 128), (4, 64, 4)):
        with pytest.raises(rl.RolaError):
            rl.ffn_workspace(rl.make_ffn_config(*bad))
