"""The stream that a call of the binding is enqueued on where the caller names none."""
import types

import torch

import paper_2403_10616_amd as dp


def test_the_current_streams_handle(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 40 + device, raising=False)
    assert dp._stream(None) == 43
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0)
    assert dp._stream(None) is None                                 # the default stream
    assert dp._stream(types.SimpleNamespace(cuda_stream=7)) == 7 and dp._stream(types.SimpleNamespace(cuda_stream=0)) is None


def test_a_torch_without_the_handles_function(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    for handle, want in ((9, 9), (0, None)):
        monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=handle))
        assert dp._stream(None) == want
