"""Which stream a call without one goes to."""
from __future__ import annotations

import pytest
import torch

from gpu_util import need_gpu
from paper_2510_02483_amd import lib as L


class Stream:
    cuda_stream = 77


def test_a_given_stream():
    assert L._stream(Stream()) == 77


def test_without_the_short_way(monkeypatch):
    """A PyTorch that does not give a stream's handle without an object for it."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    assert L._stream() == 77


@pytest.mark.gpu
def test_the_current_stream():
    need_gpu()
    assert L._stream() == torch.cuda.current_stream().cuda_stream
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert L._stream() == s.cuda_stream == torch.cuda.current_stream().cuda_stream
    g, t = torch.cuda.CUDAGraph(), torch.zeros(4, device="cuda")
    with torch.cuda.graph(g):
        assert L._stream() == torch.cuda.current_stream().cuda_stream
        t += 1
    assert L._stream() == torch.cuda.current_stream().cuda_stream != s.cuda_stream
