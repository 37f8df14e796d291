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


class On:
    """A tensor of another device, as far as the wrappers look."""

    def __init__(self, device, *shape, dtype=torch.float32):
        self.device_index, self.shape, self.dtype = device, torch.Size(shape), dtype

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        raise RuntimeError("the call went on")

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()


def parts(cache_device, batch_device):
    cache = B.QuantKV.__new__(B.QuantKV)
    cache.c, cache.head, cache.device = B.ee_quant_cache(), (2, 64), cache_device
    batch = B.ee_batch(3)
    batch.device = batch_device
    return cache, batch


@pytest.mark.parametrize("cache_device,batch_device", [(1, 0), (0, 1)])
def test_caches_and_batches_of_another_device(monkeypatch, cache_device, batch_device):
    monkeypatch.setattr(B, "_device", lambda: 0)
    cache, batch = parts(cache_device, batch_device)
    k, q, w = On(0, 3, 2, 64), On(0, 3, 4, 64), On(0, 3, 2, 40)
    kept, lens = On(0, 3, 2, 20, dtype=torch.int32), On(0, 3, dtype=torch.int32)
    for call in (lambda: B.ee_kv_quant_append(cache, 1, k, k, batch), lambda: B.ee_kv_quant_read(cache, 1, batch, k, k),
                 lambda: B.ee_paged_attention_quant(cache, 1, q, batch, q), lambda: B.ee_kv_quant_evict(cache, 1, batch, w, None, 20, 4, kept, lens)):
        with pytest.raises(AssertionError, match="current device"):
            call()
    cache, batch = parts(0, 0)
    with pytest.raises(RuntimeError, match="went on"):
        B.ee_kv_quant_append(cache, 1, k, k, batch)


def test_frequencies_of_another_device(monkeypatch):
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", lambda n, dtype, device: On(1, n, dtype=dtype))
    with pytest.raises(AssertionError, match="current device"):
        B.ee_rotary_frequencies(B.make_rotary_desc(64), device="cuda:1")


def test_what_a_batch_is_made_of(monkeypatch):
    """A batch knows its device; its tensors are on one."""
    monkeypatch.setattr(B, "_ptr", lambda t: 4096)
    lens, tables = On(1, 3, dtype=torch.int32), On(1, 3, 2, dtype=torch.int32)
    tables.dim = lambda: 2
    assert B.make_batch(None, lens, tables, 32).device == 1
    for other in (dict(tokens=On(0, 3, dtype=torch.int32)), dict(row_table=On(0, 3, dtype=torch.int32))):
        with pytest.raises(AssertionError, match="one device"):
            B.make_batch(other.get("tokens"), lens, tables, 32, other.get("row_table"))
