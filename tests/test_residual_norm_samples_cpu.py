"""The residual norm's backward of very many samples, on the CPU: its workspace holds a slot for every part and sample, the shares of
the samples are as they should be, and no index of a slot passes what an integer holds."""
import ctypes
import os
import subprocess

import pytest

from conftest import ROOT

SLOT = 3 * 4 * 4                                     # three rows of one column, padded to four floats
CSRC = os.path.join(ROOT, "paper_2609_06712_gb300", "csrc")


@pytest.fixture(scope="module")
def rl():
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


@pytest.mark.parametrize("rows", [1, 2])
@pytest.mark.parametrize("groups", [1, 31, 4863, 1 << 26, (1 << 27) + 5, 2 ** 31 - 40, 2 ** 31 - 1])
def test_the_workspace_holds_every_slot(rl, groups, rows):
    c = rl.make_residual_norm_config(groups, rows, 1)
    parts = min((groups * rows + 1) // 2, 4864)
    shares = min((groups + 31) // 32, 4096)
    need = SLOT * (parts + groups - 1)
    n = rl.library().rola_residual_norm_backward_workspace_bytes(ctypes.byref(c))
    assert need + SLOT * shares <= n <= need + SLOT * shares + 3 * 256


def test_slots_of_very_many_samples(tmp_path):
    """The offsets of a part's and a sample's sums, as the kernels take them."""
    src = tmp_path / "slots.cu"
    src.write_text('''#include <cstdio>
#include "%s"
using namespace rola;
int main() {
    for (int d : {1, 64, 1 << 20})
        for (int part : {0, 1215, 4863})
            for (int s : {0, 1 << 27, 2147483647 - 4864, 2147483646}) {
                const unsigned __int128 want = ((unsigned __int128)part + s) * 3 * ((d + 3) / 4 * 4);
                if ((unsigned __int128)rn_slot(part, s, d) != want) return 1;
            }
    puts("ok");
}''' % os.path.join(CSRC, "residual_norm.cuh"))
    from paper_2609_06712_gb300 import build
    subprocess.run([build.nvcc(), "-std=c++17", str(src), "-o", str(tmp_path / "slots")], check=True, capture_output=True)
    assert subprocess.run([str(tmp_path / "slots")], capture_output=True, text=True).stdout.strip() == "ok"


def test_the_kernels_take_their_slots_from_there():
    with open(os.path.join(CSRC, "residual_norm.cu")) as f:
        source = f.read()
    uses = [line for line in source.split("\n") if "a.part + " in line]
    assert len(uses) == 3 and all("a.part + rn_slot(" in line for line in uses)
