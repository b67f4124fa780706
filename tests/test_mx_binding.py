"""The binding of the block-scaled operators, host side: which names of torch it can do without."""
import importlib.util
import os
import types

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_binding_without_the_short_ways_into_torch(monkeypatch):
    """Device and stream come from torch's public calls where its private ones are missing."""
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=4096 + device))
    spec = importlib.util.spec_from_file_location("zr_again", os.path.join(ROOT, "paper_2401_11469_amd", "zr.py"))
    zr = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(zr)
    assert zr._here() == 3 and zr._on(None, 3) == 4099
