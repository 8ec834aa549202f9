"""Whose memory the binding's calls make their own tensors of: the stream's that the call's work runs on.  torch keeps freed memory for
each stream apart, in the order of that stream's work; memory of another's may still be read by work of that one, and is handed on to it
while the call's kernels run.  No GPU: stand-ins for torch's streams and tensors, and nothing reaches the library.
"""
import contextlib

import pytest
import torch

from paper_2410_20650_amd import binding as nz
from test_operator_arguments import ADAPTERS, BLOB, F32, I32, I64, IN, OUT, RANK, ROWS, TOKENS, Stub

CURRENT = 0x11


class Handle:
    """All that the binding asks of a stream."""

    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


class Stream(Handle):
    """Stands for torch's own class."""


@pytest.fixture
def made(monkeypatch):
    """The streams whose memory tensors are made of."""
    current, found = [CURRENT], []

    @contextlib.contextmanager
    def on(stream):
        assert isinstance(stream, Stream)
        current.append(stream.cuda_stream)
        yield
        current.pop()

    def external(handle):
        assert handle != 0
        return Stream(handle)

    def empty(*shape, dtype, device):
        shape = shape[0] if isinstance(shape[0], tuple) else shape
        found.append(current[-1])
        return Stub(shape, dtype)

    class Library:
        def __getattr__(self, name):
            return lambda *args: 512 if name.endswith("_scratch_bytes") else 0

    monkeypatch.setattr(nz, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", external)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: Stream(0))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(t.shape, dtype=t.dtype, device=t.device))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: CURRENT, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return found


STREAMS = [None, Stream(0x22), Handle(0x33), Handle(0)]
X, H, SUMS = Stub((TOKENS, IN)), Stub((TOKENS, OUT)), Stub((TOKENS, OUT), F32)
W = Stub((OUT, IN))
MANY = Stub((64, IN))     # (as many tokens as the linear layer takes scratch memory for)
ADAPTED = (Stub((ADAPTERS, RANK, IN)), Stub((ADAPTERS, OUT, RANK)), None, Stub((TOKENS,), I32), None)
WITH_SCRATCH = {
    "embedding_grad": lambda s: nz.neuzip_embedding_grad(Stub((TOKENS,), I64), X, ROWS, 1.0, Stub((ROWS, IN)), stream=s),
    "gated_linear": lambda s: nz.neuzip_gated_linear(BLOB, BLOB, OUT, IN, X, nz.SILU, H, stream=s),
    "gated_backward": lambda s: nz.neuzip_gated_backward(X, W, W, SUMS, SUMS, H, nz.SILU, X, (W, W), stream=s),
    "linear_adapters": lambda s: nz.neuzip_linear_adapters(BLOB, OUT, IN, X, *ADAPTED, SUMS, stream=s),
}


def expected(stream):
    return CURRENT if stream is None else stream.cuda_stream


@pytest.mark.parametrize("stream", STREAMS)
@pytest.mark.parametrize("name", WITH_SCRATCH)
def test_scratch_memory(made, name, stream):
    WITH_SCRATCH[name](stream)
    assert made == [expected(stream)]


# results that the caller has not brought along, and how many tensors with the scratch memory
OF_ITS_OWN = {
    "embedding": (1, lambda s: nz.neuzip_embedding(BLOB, ROWS, IN, Stub((TOKENS,), I64), stream=s)),
    "embedding_grad": (2, lambda s: nz.neuzip_embedding_grad(Stub((TOKENS,), I64), X, ROWS, stream=s)),
    "gated_linear": (2, lambda s: nz.neuzip_gated_linear(BLOB, BLOB, OUT, IN, X, stream=s)),
    "gated_forward": (1, lambda s: nz.neuzip_gated_forward(X, W, W, stream=s)),
    "gated_forward_kept": (3, lambda s: nz.neuzip_gated_forward(X, W, W, keep=True, stream=s)),
    "gated_backward": (4, lambda s: nz.neuzip_gated_backward(X, W, W, SUMS, SUMS, H, stream=s)),
    "linear_adapters": (2, lambda s: nz.neuzip_linear_adapters(BLOB, OUT, IN, X, *ADAPTED, stream=s)),
    "linear": (1, lambda s: nz.neuzip_linear(BLOB, OUT, IN, X, stream=s)),
    "linear_batch": (2, lambda s: nz.neuzip_linear_batch([BLOB, BLOB], [OUT, OUT], IN, X, stream=s)),
}


@pytest.mark.parametrize("stream", STREAMS)
@pytest.mark.parametrize("name", OF_ITS_OWN)
def test_results(made, name, stream):
    count, call = OF_ITS_OWN[name]
    call(stream)
    assert made == [expected(stream)] * count


@pytest.mark.parametrize("stream", STREAMS)
def test_results_beside_the_linear_layers_scratch_memory(made, stream):
    # (which does without, where all it has of a stream is the handle)
    nz.neuzip_linear(BLOB, OUT, IN, MANY, stream=stream)
    nz.neuzip_linear_batch([BLOB, BLOB], [OUT, OUT], IN, MANY, stream=stream)
    assert made == [expected(stream)] * (3 if type(stream) is Handle else 5)
