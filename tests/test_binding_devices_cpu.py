"""Which GPU the binding of the block operators launches on, without a GPU: stand-ins for tensors, streams, the current
device and the library's entry points."""
import contextlib

import pytest
import torch


@pytest.fixture
def rl(monkeypatch):
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    here = [0]

    @contextlib.contextmanager
    def device(d):
        before, here[0] = here[0], d if isinstance(d, int) else d.index
        yield
        here[0] = before
    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append((name, here[0], a[-1])) or 0
    monkeypatch.setattr(rola, "_lib", Lib())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: here[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 1000 + d, raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    rola.test_calls = calls
    yield rola
    del rola.test_calls


class Tensor:
    def __init__(self, shape, dtype, dev):
        self.shape, self.dtype, self.dev = torch.Size(shape), dtype, dev
        self.device, self.is_cuda = torch.device("cuda", dev) if dev >= 0 else torch.device("cpu"), dev >= 0

    def get_device(self):
        return self.dev

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 4096


class Stream:
    def __init__(self, dev):
        self.device_index, self.cuda_stream = dev, 7


BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def operators(rl):
    """name -> (function of the tensors and a stream, the tensors' shapes and dtypes)."""
    from paper_2609_06712_gb300.rola import RolaAttentionConfig, RolaFfnConfig
    f = RolaFfnConfig(tokens=4, d_model=64, d_ff=128)
    a = RolaAttentionConfig(B=2, H=4, H_kv=2, Lq=8, Lk=16, d_h=128)
    x, w, down, g = ((4, 64), BF), ((128, 64), BF), ((64, 128), BF), ((4, 128), F32)
    q, k, n, lse, ws = ((2, 4, 8, 128), BF), ((2, 2, 16, 128), BF), ((2,), I32), ((2, 4, 8), F32), ((512,), U8)
    row, vec, sums = ((4,), F32), ((64,), BF), ((64,), F32)
    return {
        "layer_norm": (lambda t, st: rl.layer_norm(t[0], t[1], t[2], 1e-6, *t[3:], stream=st), [x, vec, vec, x, row, row]),
        "layer_norm_backward": (lambda t, st: rl.layer_norm_backward(*t, stream=st), [x, vec, row, row, x, x, sums, sums, ws]),
        "ffn": (lambda t, st: rl.ffn(f, *t, stream=st), [x, w, w, down, x, ws]),
        "ffn_train": (lambda t, st: rl.ffn_train(f, *t, stream=st), [x, w, w, down, x, g, g, ws]),
        "ffn_backward": (lambda t, st: rl.ffn_backward(f, *t, stream=st), [x, w, w, down, g, g, x, x, w, w, down, ws]),
        "attention": (lambda t, st: rl.attention(a, *t, stream=st), [q, k, k, n, q, lse, ws]),
        "attention_backward": (lambda t, st: rl.attention_backward(a, *t, stream=st), [q, k, k, n, q, lse, q, q, k, k, ws]),
    }


NAMES = ["layer_norm", "layer_norm_backward", "ffn", "ffn_train", "ffn_backward", "attention", "attention_backward"]


@pytest.mark.parametrize("name", NAMES)
def test_a_call_runs_on_its_tensors_gpu(rl, name):
    call, specs = operators(rl)[name]
    for dev in (0, 1, 3):                            # GPU 0 is current
        call([Tensor(*s, dev) for s in specs], None)
        call([Tensor(*s, dev) for s in specs], Stream(dev))
        assert rl.test_calls[-2:] == [("rola_" + name, dev, 1000 + dev), ("rola_" + name, dev, 7)]
    assert torch._C._cuda_getDevice() == 0


@pytest.mark.parametrize("name", NAMES)
def test_tensors_and_streams_of_other_gpus_are_refused(rl, name):
    call, specs = operators(rl)[name]
    for i in range(len(specs)):
        for other in (1, -1):
            with pytest.raises(ValueError):
                call([Tensor(*s, other if i == j else 0) for j, s in enumerate(specs)], None)
    with pytest.raises(ValueError):
        call([Tensor(*s, -1) for s in specs], None)
    with pytest.raises(ValueError):
        call([Tensor(*s, 0) for s in specs], Stream(1))
    assert not rl.test_calls
