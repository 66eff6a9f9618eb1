"""The stream that the binding hands to the library is torch's current one, however this torch lets it be asked for."""
from types import SimpleNamespace

import pytest
import torch

from paper_2402_05109_amd import binding as hb


@pytest.mark.parametrize("missing", ["_cuda_getCurrentRawStream", "_cuda_getDevice"])
def test_without_the_names_that_are_not_public(monkeypatch, missing):
    monkeypatch.delattr(torch._C, missing, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: SimpleNamespace(cuda_stream=123))
    assert hb._pick_stream()() == 123


@pytest.mark.gpu
def test_the_current_stream_either_way(monkeypatch):
    torch.zeros(1, device="cuda:0")
    short = hb._pick_stream()
    with monkeypatch.context() as m:
        m.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
        public = hb._pick_stream()
    side = torch.cuda.Stream()
    for stream in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(stream):
            assert hb._stream() == short() == public() == stream.cuda_stream
