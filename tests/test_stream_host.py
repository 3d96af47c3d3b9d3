"""The stream that a call without one runs on: torch's current one, whether or not torch has its short way to the handle."""
import pytest

from paper_2406_14066_amd import spec_verify as sv

torch = pytest.importorskip("torch")


class _Stream:
    cuda_stream = 0x1234


@pytest.mark.parametrize("short", [True, False], ids=["raw", "object"])
def test_current_stream(monkeypatch, short):
    monkeypatch.setattr(sv, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _Stream())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    if short:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x5678 + device, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert sv._stream_handle(None) == (0x5678 + 3 if short else 0x1234)
    assert sv._stream_handle(_Stream()) == 0x1234
