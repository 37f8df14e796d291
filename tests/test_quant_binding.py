"""The Python wrappers of the 8-bit cache and the rotary embedding, on the host: what they need of torch, and what they refuse."""
import importlib.util

import pytest
import torch

from paper_2407_20272_amd import binding as B


def test_importing_needs_no_private_names(monkeypatch):
    """A torch without them (one built without GPU support) still imports the binding, and the public functions stand in."""
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("S", (), dict(cuda_stream=100 + device)))
    spec = importlib.util.spec_from_file_location("binding_without_gpu", B.__file__, submodule_search_locations=[])
    spec.loader.exec_module(m := importlib.util.module_from_spec(spec))
    assert m._device() == 3 and m._raw_stream(3) == 103
