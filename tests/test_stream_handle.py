"""The current stream's handle, with torch's function for it and without.  No GPU: stand-ins for torch's functions."""
import types

import pytest
import torch

from paper_2410_20650_amd import binding as nz


@pytest.mark.parametrize("there", [True, False])
def test_the_current_stream(monkeypatch, there):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0x77))
    if there:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x70 + device, raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert nz._stream_handle(None).value == (0x73 if there else 0x77)


def test_a_given_stream():
    assert nz._stream_handle(types.SimpleNamespace(cuda_stream=0x55)).value == 0x55
    assert nz._stream_handle(types.SimpleNamespace(cuda_stream=0)).value is None
