"""The operators on a stream that is given, with results of their own making (-m gpu): the stream as torch has it or by its handle alone, and
beside another thread's capture.
"""
import threading

import pytest
import torch

from test_gpu_operator_capture import ADAPTERS, DEV, IN, OUT, RANK, ROWS, TOKENS, bf, calls

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


class Handle:
    """All that the binding asks of a stream."""

    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


def with_results_of_its_own(nz, name):
    """The call of calls() on the same inputs, without tensors for its results."""
    if name == "embedding_grad":
        tokens, grad_out = (torch.arange(600, device=DEV) * 7) % ROWS, bf(600, IN, seed=10)
        return lambda **kw: [nz.neuzip_embedding_grad(tokens, grad_out, ROWS, 1.0, **kw)]
    x, gate, up = bf(TOKENS, IN, seed=1), bf(OUT, IN, seed=2), bf(OUT, IN, seed=3)
    if name == "gated_backward":
        g, u, gh = bf(TOKENS, OUT, seed=6).float(), bf(TOKENS, OUT, seed=7).float(), bf(TOKENS, OUT, seed=8)
        return lambda **kw: list(nz.neuzip_gated_backward(x, gate, up, g, u, gh, nz.SILU, **kw))
    blobs = [nz.neuzip_compress(w, 7) for w in (gate, up)]
    if name == "gated_linear":
        return lambda **kw: [nz.neuzip_gated_linear(*blobs, OUT, IN, x, nz.SILU, **kw)]
    ids = (torch.arange(TOKENS, device=DEV) % ADAPTERS).to(torch.int32)
    a, b = bf(ADAPTERS, RANK, IN, seed=4), bf(ADAPTERS, OUT, RANK, seed=5)
    return lambda **kw: [nz.neuzip_linear_adapters(blobs[0], OUT, IN, x, a, b, None, ids, None, **kw)]


NAMES = ["embedding_grad", "gated_linear", "gated_backward", "linear_adapters"]


def wanted(nz, name):
    call, results, apart = calls(nz)[name]
    call()
    torch.cuda.synchronize()
    return [r.clone() for r in results], apart


@pytest.mark.parametrize("kind", ["torch's", "handle", "handle 0"])
@pytest.mark.parametrize("name", NAMES)
def test_results_on_a_given_stream(nz, name, kind):
    want, apart = wanted(nz, name)
    call = with_results_of_its_own(nz, name)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        # (what the call makes for itself and drops is the stream's next tensors': nothing of it may still be needed then)
        got = call(stream={"torch's": side, "handle": Handle(side.cuda_stream), "handle 0": Handle(0)}[kind])
        torch.cuda.synchronize()
        for r, w in zip(got, want):
            assert r.shape == w.shape and (r.float() - w.float()).abs().max().item() <= apart


@pytest.mark.parametrize("name", NAMES)
def test_results_while_another_thread_captures(nz, name):
    want, apart = wanted(nz, name)
    call = with_results_of_its_own(nz, name)
    side = torch.cuda.Stream()
    count = torch.ones(1000, device=DEV)
    torch.cuda.synchronize()
    got, failed = [], []

    def other():
        try:
            got.extend(call(stream=side))
        except Exception as e:  # (told below: a thread's exception is nobody's)
            failed.append(e)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.empty_cache()
    with torch.cuda.graph(graph):   # (the global mode)
        count += 1
        thread = threading.Thread(target=other)
        thread.start()
        thread.join()
        count += 1
    assert not failed, failed
    for k in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert bool((count == 1 + 2 * k).all())
    for r, w in zip(got, want):
        assert (r.float() - w.float()).abs().max().item() <= apart
