"""CPU test of how the binding finds the current stream."""
import types

import torch

from paper_2607_02640_amd import _lib


def test_a_torch_without_the_raw_query_is_asked_for_its_stream(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert _lib._stream(None) == 103
    assert _lib._stream(5) == 5
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert _lib._stream(None) == 77
