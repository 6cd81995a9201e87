"""Which stream a call without one goes to, on the host."""
from types import SimpleNamespace

import pytest
import torch

from paper_2609_24519_b200 import binding as b


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_torch_without_the_raw_lookup(monkeypatch, missing):
    monkeypatch.delattr(torch._C, missing, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice" if missing != "_cuda_getDevice" else "_cuda_getCurrentRawStream", lambda *a: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=0x1234))
    assert b._stream(None) == 0x1234


def test_streams_that_are_named(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x100 + device, raising=False)
    assert b._stream(None) == 0x103 and b._stream(7) == 7 and b._stream(SimpleNamespace(cuda_stream=9)) == 9
