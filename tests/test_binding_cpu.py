"""The binding's own lookups, without a GPU."""
import importlib.util
import sys
import types

import torch

from paper_2510_27527_amd import binding as B


def test_stream_without_the_undocumented_lookups(monkeypatch):
    """A torch that does not have them: the documented interface gives the same stream."""
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=1000 + (3 if device is None else device)))
    spec = importlib.util.spec_from_file_location("binding_without_lookups", B.__file__)
    module = importlib.util.module_from_spec(spec)
    monkeypatch.setitem(sys.modules, spec.name, module)
    spec.loader.exec_module(module)
    assert module._stream() == 1003
