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
