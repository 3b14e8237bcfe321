"""A residual norm whose row's copy does not arrive, on the GPU: the call ends, what depends on the row is NaN, and the next call
works.  The hook leaves out each group's first copy, so that its wait runs out: that row is lost, and those that were not yet
on their way then."""
import pytest
import torch

from block_util import randn

pytestmark = pytest.mark.gpu
NAN, BF, F32 = float("nan"), torch.bfloat16, torch.float32
VECTORS = ("gate", "gamma_h", "gamma", "beta", "scale")


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


# one row; a warp a row; CTAs a row in 16-byte pieces, pairs and single elements; parts of several rows and several samples
@pytest.mark.parametrize("B,n,d,dt", [(1, 1, 64, BF), (3, 2000, 200, BF), (2, 4000, 512, F32), (2, 3001, 1536, BF), (40, 50, 1536, BF), (1, 900, 5120, BF),
                                      (2, 700, 777, F32), (2, 1500, 1537, BF), (2, 1500, 1538, BF), (1, 400, 8192, BF)])
@pytest.mark.parametrize("norm,branch,with_h", [("layer", "none", True), ("rms", "rms", True), ("layer", "layer", True), ("layer", "none", False),
                                                ("none", "none", True), ("none", "layer", True)])
def test_a_lost_row_shows(rl, norm, branch, with_h, B, n, d, dt):
    c = rl.make_residual_norm_config(B, n, d, norm, branch, dtype=rl.ROLA_BF16 if dt is BF else rl.ROLA_FP32)
    x, h, dout, dy = (randn((B, n, d), dt, i) for i in range(4))
    normed = norm != "none"
    v = dict(gate=randn((B, d), dt, 5) if with_h else None, gamma_h=randn((d,), dt, 6) if branch != "none" else None,
             gamma=randn((d,), dt, 7) if normed else None, beta=randn((d,), dt, 8) if normed else None,
             scale=randn((B, d), dt, 9) if normed else None)
    if not with_h:
        h = dout = None
    if not normed:
        dy = None
    ws = rl.residual_norm_backward_workspace(c)

    def forward():
        out, y = (torch.zeros_like(x) if there else None for there in (with_h, normed))
        stats = torch.zeros((B, n, 4), device="cuda")
        rl.residual_norm(c, x, h, out, y, stats=stats, **v)
        return out, y, stats

    def backward(stats):
        dx, dh = torch.zeros_like(x), torch.zeros_like(x) if with_h else None
        grads = {"d" + k: None if t is None else torch.zeros(t.shape, device="cuda") for k, t in v.items()}
        grads["dshift"] = torch.zeros((B, d), device="cuda") if normed else None
        rl.residual_norm_backward(c, x, h, stats, dout, dy, dx, dh, ws, **v, **grads)
        return dx, dh, *grads.values()
    want = forward()
    grads = backward(want[2])
    torch.cuda.synchronize()
    c.wait_limit_ms, c.debug_flags = 20, rl.ROLA_DEBUG_SKIP_FIRST_K_COPY
    # on the GPU's clock (the first look for NaN takes torch seconds on the host): a thread waits 20 ms once, for the last
    # copies as long again at most
    start, end = torch.cuda.Event(True), torch.cuda.Event(True)
    start.record()
    lost = forward()
    lost_grads = backward(want[2])
    end.record()
    torch.cuda.synchronize()
    assert 40 <= start.elapsed_time(end) <= 80 + 100
    rows = []                                                # a row is as it should be, or NaN
    for got, right in zip((*lost[:2], *lost_grads[:2]), (*want[:2], *grads[:2])):
        if right is not None:
            gone = torch.isnan(got).all(-1)
            assert torch.equal(got[~gone], right[~gone]) and gone[0, 0]
            rows.append(gone)
    for kind, there in ((1, normed), (3, branch != "none")):         # 1 / size of each norm
        assert not there or torch.equal(torch.isnan(lost[2][..., kind]), rows[0])
    assert all(torch.equal(gone, rows[0]) for gone in rows[:with_h + normed])
    # every sample holds the first row of a group: all sums over its rows are lost
    assert all(gone.any(-1).all() for gone in rows)
    for t in lost_grads[2:]:
        assert t is None or torch.isnan(t).all()
    c.debug_flags = 0
    for a, b in zip((*want, *grads), (*forward(), *backward(want[2]))):
        assert a is None or torch.equal(a, b)
