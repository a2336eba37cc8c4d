"""The stream that a call of the binding takes when none is given (no GPU needed)."""
from types import SimpleNamespace

import pytest
import torch

import paper_2411_06465_amd as L


@pytest.fixture
def launched(monkeypatch):
    """_launch of an entry point that keeps its arguments, on tensors of device 0 with no GPU behind them."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    tensor, seen = SimpleNamespace(device=torch.device("cuda", 0)), []

    def call(stream=None):
        L._launch(lambda *args: seen.append(args) or 0, tensor, stream, 5)
        return seen.pop()

    return call


def test_the_current_streams_handle(launched, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 1000 + index, raising=False)
    assert launched() == (5, 1000)


def test_a_torch_that_hands_out_no_bare_handles(launched, monkeypatch):
    """The public way to the same handle."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: SimpleNamespace(cuda_stream=2000 + device.index))
    assert launched() == (5, 2000)


def test_a_given_stream(launched):
    assert launched(SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=7)) == (5, 7)
    with pytest.raises(ValueError):
        launched(SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=7))
