"""Which GPU the binding of linear layers and residual norms launches on, and what it refuses, without a GPU (stand-ins as for
the other block operators)."""
import pytest
import torch

from test_binding_devices_cpu import BF, F32, U8, Stream, Tensor, rl  # noqa: F401 (rl: the fixture)


class Strided(Tensor):
    def __init__(self, shape, dtype, dev, stride=None):
        super().__init__(shape, dtype, dev)
        self.strides = stride or (shape[-1], 1)

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]


X, W, V, Y, Z, SUMS, WS = ((4, 64), BF), ((128, 64), BF), ((128,), BF), ((4, 128), BF), ((4, 128), F32), ((128,), F32), ((512,), U8)
ROWS, MOD, VEC, STATS, GMOD, GVEC = ((2, 3, 64), BF), ((2, 64), BF), ((64,), BF), ((2, 3, 4), F32), ((2, 64), F32), ((64,), F32)
VECTORS = ("gate", "gamma_h", "gamma", "beta", "scale")
GRADS = ("dgate", "dgamma_h", "dgamma", "dbeta", "dscale", "dshift")


def operators(rl):  # noqa: F811
    lin = rl.RolaLinearConfig(tokens=4, d_in=64, d_out=128)
    rn = rl.RolaResidualNormConfig(groups=2, rows=3, d=64, norm=1, branch_norm=1)
    return {
        "linear": (lambda t, st: rl.linear(lin, *t, stream=st), [X, W, V, Y, Y, WS]),
        "linear_train": (lambda t, st: rl.linear_train(lin, *t, stream=st), [X, W, V, Y, Y, Z, WS]),
        "linear_backward": (lambda t, st: rl.linear_backward(lin, *t, stream=st), [X, W, Z, Y, X, W, SUMS, WS]),
        "residual_norm": (lambda t, st: rl.residual_norm(rn, *t[:4], **dict(zip(VECTORS + ("shift", "stats"), t[4:])), stream=st),
                          [ROWS] * 4 + [MOD, VEC, VEC, VEC, MOD, MOD, STATS]),
        "residual_norm_backward": (lambda t, st: rl.residual_norm_backward(rn, *t[:8], **dict(zip(VECTORS + GRADS, t[8:])), stream=st),
                                   [ROWS, ROWS, STATS] + [ROWS] * 4 + [WS, MOD, VEC, VEC, VEC, MOD, GMOD, GVEC, GVEC, GVEC, GMOD, GMOD]),
    }


NAMES = ["linear", "linear_train", "linear_backward", "residual_norm", "residual_norm_backward"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_runs_on_its_tensors_gpu(rl, name):  # noqa: F811
    call, specs = operators(rl)[name]
    for dev in (0, 1, 3):                            # GPU 0 is current
        call([Strided(*s, dev) for s in specs], None)
        call([Strided(*s, dev) for s in specs], Stream(dev))
        assert rl.test_calls[-2:] == [("rola_" + name, dev, 1000 + dev), ("rola_" + name, dev, 7)]
    assert torch._C._cuda_getDevice() == 0


@pytest.mark.parametrize("name", NAMES)
def test_tensors_and_streams_of_other_gpus_are_refused(rl, name):  # noqa: F811
    call, specs = operators(rl)[name]
    for i in range(len(specs)):
        for other in (1, -1):
            with pytest.raises(ValueError):
                call([Strided(*s, other if i == j else 0) for j, s in enumerate(specs)], None)
    with pytest.raises(ValueError):
        call([Strided(*s, 0) for s in specs], Stream(1))
    assert not rl.test_calls


def test_vectors_of_other_strides_are_refused(rl):  # noqa: F811
    c = rl.RolaResidualNormConfig(groups=2, rows=3, d=64, norm=1, mod_stride=384)
    t = [Strided(*ROWS, 0) for _ in range(4)]
    rl.residual_norm(c, *t, gate=Strided(*MOD, 0, (384, 1)))
    for stride in ((64, 1), (384, 2), (0, 1)):
        for name in ("gate", "scale", "shift"):
            with pytest.raises(ValueError):
                rl.residual_norm(c, *t, **{name: Strided(*MOD, 0, stride)})
    assert len(rl.test_calls) == 1


def test_slices_of_one_modulation_stay_where_they_are(rl):  # noqa: F811
    mod = torch.randn(3, 6, 8)
    a, b, none, apart = rl._same_stride((mod[:, 1], mod[:, 4], None), 8)
    assert apart == 48 and none is None and a.data_ptr() == mod[:, 1].data_ptr() and b.data_ptr() == mod[:, 4].data_ptr()
    for vectors in ((mod[:, 1], torch.randn(3, 8)), (mod[:, 1], mod.transpose(1, 2).contiguous()[:, :, 0]), (torch.randn(8).expand(3, 8),)):
        *made, apart = rl._same_stride(vectors, 8)
        assert apart == 8 and all(t.is_contiguous() and torch.equal(t, v) for t, v in zip(made, vectors))
    assert rl._same_stride((None, mod[:1, 2], None), 8)[3] == 8
