"""Group norm and AdamW when another device than their handle's or their tensors' is current: refused on the host, without a GPU."""
import ctypes

import pytest
import torch

from paper_2104_06700_b200 import binding
from test_host_side import fake, library  # noqa: F401
from test_norm_host import calls


def test_a_handle_of_another_device_is_refused(fake):  # noqa: F811
    g = fake.graph(64, 256)
    bad = binding.DG_ERR_INVALID_ARG
    fake.lib.cudaSetDevice(1)
    fake.events()
    assert calls(fake, g) == (bad, bad) and b"device" in fake.lib.dg_last_error()
    assert fake.events() == []
    offsets = (ctypes.c_int64 * 3)(0, 10, 64)      # moves to the handle's by itself
    assert fake.lib.dg_graph_set_batch(g, ctypes.c_int64(2), offsets) == binding.DG_OK
    device = ctypes.c_int()
    fake.lib.cudaGetDevice(ctypes.byref(device))
    assert device.value == 1
    fake.lib.cudaSetDevice(0)
    assert calls(fake, g) == (binding.DG_OK, binding.DG_OK)
    fake.lib.dg_graph_destroy(g)


def test_a_list_of_another_device_is_refused(monkeypatch):
    class Library:
        def __getattr__(self, name):
            def call(*_):
                raise AssertionError("called")
            return call

    monkeypatch.setattr(binding, "lib", Library)
    monkeypatch.setattr(binding, "_check_tensors", lambda tensors, dtypes, device, name: [t.dtype for t in tensors])
    monkeypatch.setattr(binding, "_device", lambda: 1)
    grads = [torch.zeros(5)]
    a = binding.AdamwList(grads, [torch.zeros(5)], [torch.zeros(5)], [torch.zeros(5)], [torch.zeros((), dtype=torch.int64)])
    a.device = 0           # made while the first device was current
    ws, result = torch.zeros(binding.DG_ADAMW_WORKSPACE_BYTES, dtype=torch.uint8), torch.zeros(2)
    with pytest.raises(ValueError, match="device"):
        binding.dg_grad_norm(a, 1.0, ws, result)
    with pytest.raises(ValueError, match="device"):
        binding.dg_adamw_step(a, 1e-3, 0.9, 0.999, 1e-8, 0.0, ws)
    a.device = 1           # then the call goes on to its other checks
    with pytest.raises(ValueError, match="CUDA"):
        binding.dg_grad_norm(a, 1.0, ws, result)
