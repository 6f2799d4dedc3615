"""The binding's choice of a stream, on the host."""
from types import SimpleNamespace

from paper_2510_01565_amd import dit


def test_current_stream_with_and_without_torchs_raw_handle(monkeypatch):
    """A torch without the private call for the raw handle is asked for the stream's object."""
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=7))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 10 + device, raising=False)
    assert dit._stream(None) == 13
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert dit._stream(None) == 7


def test_given_streams_pass_as_they_are():
    assert dit._stream(0) == 0 and dit._stream(5) == 5 and dit._stream(SimpleNamespace(cuda_stream=9)) == 9
