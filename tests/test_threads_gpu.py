"""Calls of several host threads at once, of the same kernels at sizes that need different amounts of shared memory: each
succeeds and gives the bits that it gives alone."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rl():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    return rola


def rand(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def together(makers, rounds):
    """makers: functions that return (call, its output).  Runs each call `rounds` times in a thread and stream of its own."""
    made = [m() for m in makers]
    alone = []
    for call, out in made:
        call(torch.cuda.current_stream())
        torch.cuda.synchronize()
        alone.append(out.clone())
    errors, start = [], threading.Barrier(len(made))

    def work(call, stream):
        try:
            start.wait()
            for _ in range(rounds):
                call(stream)
        except Exception as e:                       # noqa: BLE001 (reported by the test's thread)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(call, torch.cuda.Stream())) for call, _ in made]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors[:3]
    for (_, out), want in zip(made, alone):
        assert torch.equal(out, want)


def test_layer_norm(rl):
    def maker(d):
        def make():
            x = rand(1000, d, seed=d)
            y = torch.empty_like(x)
            return lambda st: rl.layer_norm(x, None, None, 1e-6, y, stream=st), y
        return make
    together([maker(12288), maker(16384), maker(13000)], 4000)


def test_feed_forward_of_few_tokens(rl):
    def maker(m):
        def make():
            X, Wg, Wu, Wd = rand(m, 256), rand(512, 256, seed=1), rand(512, 256, seed=2), rand(256, 512, seed=3)
            c, Y = rl.make_ffn_config(m, 256, 512), torch.empty_like(X)
            ws = rl.ffn_workspace(c)
            return lambda st: rl.ffn(c, X, Wg, Wu, Wd, Y, ws, stream=st), Y
        return make
    together([maker(1), maker(96), maker(40)], 4000)
