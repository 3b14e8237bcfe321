"""Shared by the tests of the block operators: 64-bit references with their rounding bounds, and directional
differences.

Bounds are elementwise and first order.  With u = 2^-8 the unit roundoff of bf16 (8 significant bits: round to nearest
is within half of the spacing 2^-7), an output rounded once is within u |ref| of the value it rounds; an operand of a product rounded
once moves the product by at most u times the same product of absolute values; a sum of n fp32 products is within
n 2^-24 of the same sum of absolute values, for any order.  Elementary functions are within a few fp32 units of
roundoff: E = 2^-20 covers them and the handful of fp32 operations around a product.
"""
import torch

U16 = 2.0 ** -8
U32 = 2.0 ** -24
E = 2.0 ** -20
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def randn(shape, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(dtype).cuda()


def within(name, got, ref, bound):
    """|got - ref| <= bound everywhere; both finite."""
    err = (got.double() - ref).abs()
    assert torch.isfinite(got).all(), f"{name}: not finite"
    if err.numel():
        worst = (err / (bound + 1e-300)).max().item()
        assert (err <= bound).all(), f"{name}: {worst:.3f} of the bound, max error {err.max().item():.3e}"


def out_u(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def directional(f, x, d):
    """Central differences of the scalar f at x along d with steps h and h / 2: (extrapolated, their gap)."""
    def slope(h):
        return (f(x + h * d) - f(x - h * d)) / (2 * h)
    a, b = slope(2.0 ** -5), slope(2.0 ** -6)
    return (4 * b - a) / 3, abs(a - b)
