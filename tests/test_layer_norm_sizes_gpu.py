"""Layer norm at sizes whose ring of rows comes close to the 48 KB that a kernel may have without asking for more, and
at rows enough that each ring is refilled many times."""
import pytest
import torch

import test_layer_norm_gpu as base
from block_util import DTYPES

pytestmark = pytest.mark.gpu
rl = base.rl


# rings of 48512 to 49152 bytes: two rows of 24 KB, three of 16 KB x 2 in the backward, and neighbours
@pytest.mark.parametrize("rows,d,dname", [
    (100, 12136, "bf16"), (100, 12224, "bf16"), (100, 12256, "bf16"), (100, 12264, "bf16"), (100, 6112, "fp32"),
    (700, 4048, "bf16"), (700, 4080, "bf16"), (700, 2024, "fp32"), (700, 2040, "fp32")])
def test_rings_of_48_kb(rl, rows, d, dname):
    x, gamma, beta, dy = base.inputs_of(rows, d, DTYPES[dname], seed=d)
    base.check(x, gamma, beta, dy, base.run(rl, x, gamma, beta, dy))


# every CTA or warp takes tens of rows: warps (64, 512), CTAs with deep and shallow rings, single elements
@pytest.mark.parametrize("rows,d", [(100000, 64), (60001, 512), (20000, 1536), (6000, 5120), (3000, 12224), (9000, 777), (3000, 4999)])
@pytest.mark.parametrize("dname", sorted(DTYPES))
def test_many_rows(rl, rows, d, dname):
    if dname == "fp32" and d == 12224:
        d //= 2
    x, gamma, beta, dy = base.inputs_of(rows, d, DTYPES[dname], seed=d)
    got = base.run(rl, x, gamma, beta, dy)
    base.check(x, gamma, beta, dy, got)
    again = base.run(rl, x, gamma, beta, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("offset", [1000.3, -54321.7])
@pytest.mark.parametrize("d", [777, 1536])
def test_offsets_whose_mean_is_rounded(rl, offset, d):
    """The mean of such rows is not an fp32 number: x - mu carries its rounding, |mu| d 2^-24 at most, which check's bounds
    hold; the variance, about that mean, does not cancel."""
    x, gamma, beta, dy = base.inputs_of(200, d, DTYPES["fp32"], seed=d)
    x = x + offset
    got = base.run(rl, x, gamma, beta, dy)
    base.check(x, gamma, beta, dy, got)
    # a row's sum is at most 18 additions deep (8 or 9 in a thread, 5 in a warp, 3 to 5 across warps), its mean two
    # roundings more, each within 2^-24 of |mu|; what else happens is within 2^-18 of y
    rstd = (x.double().var(1, unbiased=False, keepdim=True) + base.EPS).rsqrt()
    y = (x.double() - x.double().mean(1, keepdim=True)) * rstd * gamma.double() + beta.double()
    bound = 20 * 2.0 ** -24 * (abs(offset) + 4) * rstd * gamma.double().abs() + 2.0 ** -18 * (1 + y.abs())
    assert ((got[0].double() - y).abs() <= bound).all()
