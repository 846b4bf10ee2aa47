"""Calls of the binding without a GPU: tensors of the host that say they are on a CUDA device, and a
library that records its arguments instead of launching anything.

What is tested this way is what the binding decides: what it refuses, copies, allocates and passes on.
"""

import types

import torch

from paper_2609_36246_gb300 import binding as B
from paper_2609_36246_gb300 import build


class Recorder:
    """A library whose entry points do nothing, say OLIVE_OK and keep their arguments; what
    they would have written reads 1.

    Tensors are on device 0, the current one, except those that place() put elsewhere."""

    def __init__(self):
        build.build()
        self.calls = []
        self._index = {}
        # (host checks are the library's own)
        self.olive_grad_clip_apart = B.lib().olive_grad_clip_apart

    def place(self, t, index):
        self._index[id(t)] = (index, t)  # (t is held, so that its id stays its own)
        return t

    def device_index(self, t):
        return self._index.get(id(t), (0,))[0]

    def __getattr__(self, name):
        def call(*args):
            if name == "olive_workspace_size":
                return 256
            self.calls.append(types.SimpleNamespace(name=name, args=args))
            return 0

        return call

    def named(self, name):
        return [c.args for c in self.calls if c.name == name]


def recorded(monkeypatch):
    """The recorder that stands in for the library until the test ends."""
    rec = Recorder()
    monkeypatch.setattr(B, "lib", lambda: rec)
    monkeypatch.setattr(B, "_ws_bytes", lambda *_: 256)
    monkeypatch.setattr(B, "_device_of", rec.device_index)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_current", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: rec.device_index(t))
    monkeypatch.setattr(torch.Tensor, "device", property(lambda t: torch.device("cuda", rec.device_index(t))))
    # (what is allocated on a CUDA device lies on the host)
    for name, real in (("empty", torch.ones), ("ones", torch.ones), ("zeros", torch.zeros)):
        monkeypatch.setattr(torch, name, lambda *a, _real=real, device=None, **k: _real(*a, **k))
    return rec
