"""Infinite and undefined sums of a linear layer on the GPU: every form (by tokens, by dtype) gives the feature map's own
value, and what is not finite stays in its row."""
import pytest
import torch

from block_util import DTYPES, randn

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
# phi and phi' at (inf, -inf, nan), as their formulas give them: g / (1 + e^-g) and g erfc(-g / sqrt 2) / 2 are -inf / inf and
# -inf * 0 at -inf, and their slopes have an infinity times 0 at both ends
PHI = {"identity": (INF, -INF, NAN), "silu": (INF, NAN, NAN), "tanh": (1.0, -1.0, NAN), "relu": (INF, 0.0, NAN), "gelu": (INF, NAN, NAN)}
SLOPE = {"identity": (1.0, 1.0, 1.0), "silu": (NAN, NAN, NAN), "tanh": (0.0, 0.0, NAN), "relu": (1.0, 0.0, NAN), "gelu": (NAN, NAN, NAN)}
K, N = 264, 520


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def same(got, want):
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])


# weight rows up to 4 tokens, weight tiles up to 672 (one of 96, then several), tiles of pairs; fp32: rows up to 32, tiles
@pytest.mark.parametrize("m", [1, 4, 5, 33, 96, 97, 672, 673, 2000])
@pytest.mark.parametrize("dname", sorted(DTYPES))
@pytest.mark.parametrize("act", sorted(PHI))
def test_sums_that_are_not_finite(rl, act, dname, m):
    dt = DTYPES[dname]
    c = rl.make_linear_config(m, K, N, act, rl.ROLA_BF16 if dt == torch.bfloat16 else rl.ROLA_FP32)
    X, W, b, dY = randn((m, K), dt, 1), randn((N, K), dt, 2, K ** -0.5), randn((N,), dt, 3, 0.3), randn((m, N), dt, 4).abs() + 0.5
    W[:, 100] = torch.where(torch.arange(N, device="cuda") % 2 == 0, 1.0, -1.0).to(dt)
    ws, bws = rl.linear_workspace(c), rl.linear_backward_workspace(c)

    def run():
        Y, kept, Z, db = torch.empty_like(dY), torch.empty_like(dY), torch.empty((m, N), device="cuda"), torch.empty((N,), device="cuda")
        rl.linear(c, X, W, b, None, Y, ws)
        rl.linear_train(c, X, W, b, None, kept, Z, ws)
        rl.linear_backward(c, X, W, Z, dY, None, None, db, bws)
        assert same(Y, kept), "the training forward gives other values"
        return Y, Z, db
    clean, row = run(), m // 2
    for value in (INF, NAN):
        X[row, 100] = value
        Y, Z, db = run()
        # inf: the even columns' sums are inf, the odd ones' -inf
        kinds = [0, 1] if value == INF else [2, 2]
        for column, kind in enumerate(kinds):
            z = torch.full((N // 2,), (INF, -INF, NAN)[kind], device="cuda")
            assert same(Z[row, column::2], z)
            assert same(Y[row, column::2].float(), torch.full_like(z, PHI[act][kind]))
            d = dY[row, column::2].float() * SLOPE[act][kind]
            if m == 1:
                assert same(db[column::2], d)
            else:
                assert torch.equal(torch.isnan(db[column::2]), torch.isnan(d))
        others = torch.arange(m, device="cuda") != row
        assert torch.equal(Y[others], clean[0][others]) and torch.equal(Z[others], clean[1][others])
