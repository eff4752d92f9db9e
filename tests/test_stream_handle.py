"""The stream that the binding's helper passes on: the current one of the current
device, also with a torch that lacks the direct read."""
import types

import pytest
import torch

from paper_2510_16292_amd import binding as B


def stream(handle):
    return types.SimpleNamespace(cuda_stream=handle)


def test_given_stream():
    assert B.stream_handle(stream(7)) == 7


def test_current_stream_of_the_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert B.stream_handle() == 103


def test_torch_without_the_direct_read(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: stream(42))
    assert B.stream_handle() == 42


@pytest.mark.gpu
def test_handles_are_those_of_torch(monkeypatch):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert B.stream_handle() == side.cuda_stream == torch.cuda.current_stream().cuda_stream
    assert B.stream_handle() == torch.cuda.current_stream().cuda_stream
    assert B.stream_handle(side) == side.cuda_stream
    with monkeypatch.context() as m, torch.cuda.stream(side):
        m.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
        assert B.stream_handle() == side.cuda_stream
