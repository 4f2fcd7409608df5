"""Which stream a call without one goes to."""
import types

import torch

import paper_2506_21263_amd as dlcx


def test_the_current_stream_does_not_hang_on_a_private_name_of_torch(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=77))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(dlcx, "_raw_stream", None)
    assert dlcx._stream(None) == 77
    monkeypatch.setattr(dlcx, "_raw_stream", lambda device: 100 + device)
    assert dlcx._stream(None) == 103
    assert dlcx._stream(5) == 5 and dlcx._stream(types.SimpleNamespace(cuda_stream=6)) == 6
