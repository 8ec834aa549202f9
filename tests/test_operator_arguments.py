"""What the operators' calls refuse without a GPU: the binding by the tensors it is given (stand-ins, and nothing reaches the library), the
library by its arguments, before any device work.
"""
import ctypes
import math
import types

import pytest
import torch

from paper_2410_20650_amd import binding as nz

BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


class Stub:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype=BF, cuda=True, contiguous=True):
        self.shape, self.dtype, self.is_cuda, self.device = tuple(shape), dtype, cuda, "cuda:0"
        self._contiguous = contiguous

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def is_contiguous(self):
        return self._contiguous

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 0x1000


BLOB = types.SimpleNamespace(handle=ctypes.c_void_p(0x2000))
SCRATCH = Stub((1 << 20,), torch.uint8)
TOKENS, IN, OUT, ROWS, RANK, ADAPTERS = 3, 256, 40, 50, 16, 4


def embedding(tokens=Stub((TOKENS,), I64), out=Stub((TOKENS, IN))):
    nz.neuzip_embedding(BLOB, ROWS, IN, tokens, 1.0, out)


def embedding_grad(tokens=Stub((TOKENS,), I64), grad_out=Stub((TOKENS, IN)), grad=Stub((ROWS, IN)), scratch=SCRATCH):
    nz.neuzip_embedding_grad(tokens, grad_out, ROWS, 1.0, grad, scratch)


def gated_linear(x=Stub((TOKENS, IN)), h=Stub((TOKENS, OUT)), scratch=SCRATCH):
    nz.neuzip_gated_linear(BLOB, BLOB, OUT, IN, x, nz.SILU, h, scratch)


def gated_forward(x=Stub((TOKENS, IN)), w_gate=Stub((OUT, IN)), w_up=Stub((OUT, IN)), h=Stub((TOKENS, OUT)),
                  keep=(Stub((TOKENS, OUT), F32), Stub((TOKENS, OUT), F32))):
    nz.neuzip_gated_forward(x, w_gate, w_up, nz.SILU, h, keep)


def gated_backward(x=Stub((TOKENS, IN)), w_gate=Stub((OUT, IN)), gate=Stub((TOKENS, OUT), F32), grad_h=Stub((TOKENS, OUT)),
                   grad_x=Stub((TOKENS, IN)), grad_weights=(Stub((OUT, IN)), Stub((OUT, IN))), scratch=SCRATCH):
    nz.neuzip_gated_backward(x, w_gate, Stub((OUT, IN)), gate, Stub((TOKENS, OUT), F32), grad_h, nz.SILU, grad_x, grad_weights, scratch)


def adapters(x=Stub((TOKENS, IN)), a=Stub((ADAPTERS, RANK, IN)), b=Stub((ADAPTERS, OUT, RANK)), scales=Stub((ADAPTERS,), F32),
             ids=Stub((TOKENS,), I32), bias=Stub((OUT,), F32), y=Stub((TOKENS, OUT), F32), scratch=SCRATCH):
    nz.neuzip_linear_adapters(BLOB, OUT, IN, x, a, b, scales, ids, bias, y, scratch)


CALLS = {
    embedding: dict(tokens=((TOKENS,), I64), out=((TOKENS, IN), BF)),
    embedding_grad: dict(tokens=((TOKENS,), I64), grad_out=((TOKENS, IN), BF), grad=((ROWS, IN), BF)),
    gated_linear: dict(x=((TOKENS, IN), BF), h=((TOKENS, OUT), BF)),
    gated_forward: dict(x=((TOKENS, IN), BF), w_gate=((OUT, IN), BF), w_up=((OUT, IN), BF), h=((TOKENS, OUT), BF)),
    gated_backward: dict(x=((TOKENS, IN), BF), w_gate=((OUT, IN), BF), gate=((TOKENS, OUT), F32), grad_h=((TOKENS, OUT), BF),
                         grad_x=((TOKENS, IN), BF)),
    adapters: dict(x=((TOKENS, IN), BF), a=((ADAPTERS, RANK, IN), BF), b=((ADAPTERS, OUT, RANK), BF), scales=((ADAPTERS,), F32),
                   ids=((TOKENS,), I32), bias=((OUT,), F32), y=((TOKENS, OUT), F32)),
}


@pytest.fixture
def called(monkeypatch):
    """The names of the library's functions that are called."""
    names = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: names.append(name) or 0

    monkeypatch.setattr(nz, "_lib", Library())
    monkeypatch.setattr(nz, "_stream_handle", lambda stream: None)
    return names


@pytest.mark.parametrize("call", CALLS)
def test_accepted(called, call):
    call()
    assert [n for n in called if not n.endswith("_scratch_bytes")] == ["neuzip_" + {"adapters": "linear_adapters"}.get(call.__name__, call.__name__)]


@pytest.mark.parametrize("call,name", [(c, n) for c, names in CALLS.items() for n in names])
def test_refused(called, call, name):
    shape, dtype = CALLS[call][name]
    bad = [(TypeError, Stub(shape, torch.float64)), (TypeError, Stub(shape, dtype, cuda=False)), (TypeError, Stub(shape, dtype, contiguous=False)),
           (ValueError, Stub((*shape[:-1], shape[-1] + 1), dtype))]
    for error, stub in bad:
        if error is ValueError and (call, name) == (embedding, "tokens"):
            continue    # (any number of tokens will do, and then it is the output that does not fit)
        with pytest.raises(error):
            call(**{name: stub})
    assert [n for n in called if not n.endswith("_scratch_bytes")] == []


@pytest.mark.parametrize("call", [embedding_grad, gated_linear, gated_backward, adapters])
def test_scratch_memory(called, call):
    for stub in (Stub((64,), torch.uint8, cuda=False), Stub((64,), torch.uint8, contiguous=False)):
        with pytest.raises(TypeError):
            call(scratch=stub)
    assert [n for n in called if not n.endswith("_scratch_bytes")] == []


def test_the_library_refuses_before_any_device_work():
    lib, null, some, odd = nz.library(), None, ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
    forward, backward = lib.neuzip_gated_forward, lib.neuzip_gated_backward
    for args in ((some, some, some, 3, 40, 250, 0, some, null, null), (some, some, some, 3, 0, 256, 0, some, null, null),
                 (some, some, some, 3, 40, 256, 2, some, null, null), (some, some, some, 3, 40, 256, -1, some, null, null),
                 (null, some, some, 3, 40, 256, 0, some, null, null), (some, some, some, 3, 40, 256, 0, null, null, null),
                 (some, some, some, 3, 40, 256, 0, some, some, null), (odd, some, some, 3, 40, 256, 0, some, null, null),
                 (some, some, some, 1 << 31, 40, 256, 0, some, null, null), (some, some, some, 3, 40, 1 << 23, 0, some, null, null)):
        assert forward(*args, None) == nz.EINVAL, args
    assert forward(null, null, null, 0, 40, 256, 0, null, null, null, None) == nz.OK       # no tokens: nothing to do
    room = lib.neuzip_gated_backward_scratch_bytes(3, 40, 256)
    assert room >= 2 * 3 * 40 * 2
    for args in ((some,) * 6 + (3, 40, 256, 0, some, some, some, some, room - 1), (some,) * 6 + (3, 40, 256, 0, some, some, null, some, room),
                 (some,) * 5 + (null, 3, 40, 256, 0, some, some, some, some, room), (null,) + (some,) * 5 + (3, 40, 256, 0, some, some, some, some, room),
                 (some,) * 6 + (3, 40, 256, 0, odd, some, some, some, room)):
        assert backward(*args, None) == nz.EINVAL, args
    grad = lib.neuzip_embedding_grad
    room = lib.neuzip_embedding_grad_scratch_bytes(600, 50, 256)
    assert room > 0
    for args in ((some, 600, some, 50, 250, 1.0, some, some, room + 4096), (some, 600, some, 0, 256, 1.0, some, some, room),
                 (some, 600, some, 50, 256, 1.0, null, some, room), (some, 600, some, 50, 256, 1.0, odd, some, room),
                 (null, 600, some, 50, 256, 1.0, some, some, room), (some, 600, some, 50, 256, 1.0, some, some, room - 1),
                 (some, 600, some, 1 << 24, 256, 1.0, some, some, room)):
        assert grad(*args, None) == nz.EINVAL, args
    assert grad(some, 1 << 31, some, 50, 256, 1.0, some, some, room, None) == nz.EUNSUPPORTED
    # something that is not a blob
    assert lib.neuzip_embedding(null, 50, 256, some, 3, 1.0, some, None) == nz.EINVAL
    assert lib.neuzip_gated_linear(null, null, 40, 256, some, 3, 0, some, some, 1 << 30, None) == nz.EINVAL
    assert lib.neuzip_linear_adapters(null, 40, 256, some, 3, null, some, some, 16, 4, null, some, some, some, 1 << 30, None) == nz.EINVAL
    for rank in (0, 12, 520):
        assert lib.neuzip_linear_adapters(null, 40, 256, some, 3, null, some, some, rank, 4, null, some, some, some, 1 << 30, None) == nz.EINVAL


def test_scratch_memory_of_odd_shapes_is_none():
    assert nz.neuzip_embedding_grad_scratch_bytes(512, 50, 256) == 0 and nz.neuzip_embedding_grad_scratch_bytes(64, 128256, 4096) == 0   # (in one launch)
    assert nz.neuzip_embedding_grad_scratch_bytes(513, 50, 256) > 0 and nz.neuzip_embedding_grad_scratch_bytes(65, 128256, 4096) > 0
    assert nz.neuzip_embedding_grad_scratch_bytes(0, 50, 256) == 0 and nz.neuzip_embedding_grad_scratch_bytes(10, 50, 250) == 0
    assert nz.neuzip_gated_backward_scratch_bytes(0, 40, 256) == 0 and nz.neuzip_gated_backward_scratch_bytes(3, 41, 256) == 0
