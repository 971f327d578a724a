"""The stream that the binding hands to the library when none is named: the current one, with or without
torch's shortcut to its handle."""
import types

import pytest
import torch

import paper_2607_05439_amd as dcp


def without_shortcut(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)


def test_without_torch_s_shortcut(monkeypatch):
    without_shortcut(monkeypatch)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0x1230))
    assert dcp._stream(None) == 0x1230
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0))
    assert dcp._stream(None) is None


def test_a_named_stream():
    assert dcp._stream(0x40) == 0x40 and dcp._stream(0) is None
    assert dcp._stream(types.SimpleNamespace(cuda_stream=0x50)) == 0x50


@pytest.mark.gpu
def test_the_current_stream(monkeypatch):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert dcp._stream(None) == side.cuda_stream
    assert dcp._stream(None) == (torch.cuda.current_stream().cuda_stream or None)
    without_shortcut(monkeypatch)
    with torch.cuda.stream(side):
        assert dcp._stream(None) == side.cuda_stream
