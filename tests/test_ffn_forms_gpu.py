"""The feed-forward takes the form of its products that suits the tokens: more tokens at the same widths do not make a
call faster.  (A rule that looked at the down product's tiles alone kept tiles of few tokens side by side up to 9600
tokens, where they take 1.6 to 2.4 times as long.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fewer,more,d,f", [(4500, 5000, 512, 8192), (1500, 1700, 1536, 4096), (9600, 9900, 64, 4096)])
def test_fewer_tokens_take_no_longer(fewer, more, d, f):
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import rola
    Wg, Wu, Wd = (torch.randn(s, device="cuda").bfloat16() for s in ((f, d), (f, d), (d, f)))

    def call(m):
        X = torch.randn(m, d, device="cuda").bfloat16()
        c, Y = rola.make_ffn_config(m, d, f), torch.empty_like(X)
        ws = rola.ffn_workspace(c)
        return lambda: rola.ffn(c, X, Wg, Wu, Wd, Y, ws)
    calls, best = (call(fewer), call(more)), [1e9, 1e9]
    for _ in range(10):                              # in turn, the best of ten groups of ten
        for i, go in enumerate(calls):
            go()
            a, b = torch.cuda.Event(True), torch.cuda.Event(True)
            a.record()
            for _ in range(10):
                go()
            b.record()
            torch.cuda.synchronize()
            best[i] = min(best[i], a.elapsed_time(b))
    assert best[0] <= 1.3 * best[1], best
