"""The DiT block runs on its input's GPU whatever the current one is (stand-ins for both)."""
import contextlib

import torch


def test_forward_makes_its_inputs_gpu_current(monkeypatch):
    from paper_2609_06712_gb300 import build
    build.build()
    from paper_2609_06712_gb300 import dit_block
    here = [torch.device("cuda", 0)]

    @contextlib.contextmanager
    def device(d):
        before, here[0] = here[0], d
        yield
        here[0] = before

    class Input:
        device = torch.device("cuda", 1)

        def view(self, *_):
            raise LookupError

    def linear(*_):
        seen.append(here[0])
        raise LookupError
    seen = []
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(dit_block, "linear", linear)
    block = object.__new__(dit_block.DiTBlock)
    torch.nn.Module.__init__(block)
    block.W_qkv = None
    block._norm = lambda i, x: x
    with contextlib.suppress(LookupError):
        block.forward(Input(), None)
    assert seen == [torch.device("cuda", 1)]
