"""CPU tests of the Python binding around the C entry points: streams, and a gradient
list's memory.  The library's launches are replaced by stand-ins, tensors by objects
with an address."""
import ctypes

import pytest
import torch

import paper_2606_19528_amd as lm
from paper_2606_19528_amd import lora as L


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


def test_current_stream_without_the_raw_query(monkeypatch):
    """The current stream's handle is found where torch has no function that returns it alone."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: _Stream(0x1230))
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert L._stream(None).value == 0x1230
    assert L._stream(_Stream(0x4560)).value == 0x4560
