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


class _Buffer:
    """What the binding reads of a GPU tensor."""
    is_cuda, device, dtype = True, "cpu", torch.float32

    def __init__(self, address, n, dtype=torch.float32):
        self.address, self.n, self.dtype, self.shape = address, n, dtype, torch.Size([n])
        self.recorded = []

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.n

    def element_size(self):
        return 2 if self.dtype == torch.bfloat16 else 4

    def is_contiguous(self):
        return True

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


@pytest.fixture
def launches(monkeypatch):
    """Names of the list's calls that reach the library; the current stream is 0x10."""
    names = []

    class Library:
        def grad_list_bytes(self, grads, n):
            return 8192

        def __getattr__(self, name):
            def call(*args):
                names.append(name)
                return 0
            return call

    monkeypatch.setattr(L, "lib", lambda: Library())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: _Stream(0x10))
    monkeypatch.setattr(L, "_stream", lambda s: ctypes.c_void_p((s or _Stream(0x10)).cuda_stream))
    monkeypatch.setattr(L, "_ws", lambda ws, n, like, stream=None: (_Buffer(0x900000, n, torch.uint8), n))
    return names


BF16 = torch.bfloat16


@pytest.mark.parametrize("at,n,fits", [
    (0x100000, 1, False), (0x100ffc, 1, False), (0x0ffffc, 2, False), (0x0ffffc, 1, True), (0x0ffff8, 2, True),
    (0x101000, 2, True),                                                              # a gradient's 4096 bytes
    (0x200000, 2, False), (0x2007fc, 1, False), (0x200800, 2, True), (0x1ffffc, 2, False),  # an output's 2048
    (0x300000, 1, False), (0x301ffc, 2, False), (0x302000, 2, True),                  # clipped in place
    (0x400000, 2, False), (0x402ffc, 1, False), (0x403000, 1, True),                  # gradients that overlap
])
def test_norm_apart_from_the_listed_gradients(launches, at, n, fits):
    """A norm inside a gradient or an output would be written while others read there."""
    grads = [_Buffer(0x300000, 2048), _Buffer(0x100000, 1024), _Buffer(0x500000, 0), _Buffer(0x400000, 2048),
             _Buffer(0x401000, 2048)]
    outs = [grads[0], _Buffer(0x200000, 1024, BF16), grads[2], _Buffer(0x600000, 2048), _Buffer(0x700000, 2048)]
    gl = lm.grad_list(grads, outs)
    del launches[:]

    def call():
        return lm.grad_norm(gl, _Buffer(at, 1)) if n == 1 else lm.grad_clip(gl, 1.0, _Buffer(at, 2))

    if fits:
        call()
        assert len(launches) == 1
    else:
        with pytest.raises(lm.LoraError):
            call()
        assert not launches


def test_list_memory_stays_while_another_stream_uses_it(launches):
    """The list's own memory is allocated on the stream that lays it out.  A call on another
    stream has to tell the allocator, or the memory of a list that is dropped goes to
    another tensor while that stream's kernels still read addresses from it."""
    gl = lm.grad_list([_Buffer(0x100000, 1024)], stream=_Stream(0x10))
    lm.grad_clip(gl, 1.0, _Buffer(0x800000, 2))
    lm.grad_norm(gl, _Buffer(0x800000, 1), stream=_Stream(0x10))
    assert gl.mem.recorded == []  # its own stream
    lm.grad_clip(gl, 1.0, _Buffer(0x800000, 2), stream=_Stream(0x20))
    lm.grad_norm(gl, _Buffer(0x800000, 1), stream=_Stream(0x30))
    assert gl.mem.recorded == [0x20, 0x30]
    other = lm.grad_list([_Buffer(0x100000, 1024)], stream=_Stream(0x20))
    lm.grad_clip(other, 1.0, _Buffer(0x800000, 2))  # the current stream
    assert other.mem.recorded == [0x10]
