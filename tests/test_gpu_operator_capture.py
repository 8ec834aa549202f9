"""The operators' own scratch memory and another thread's capture, and calls of more work than a launch has room for (-m gpu)."""
import ctypes
import threading

import pytest
import torch

from paper_2410_20650_amd import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOKENS, IN, OUT, ROWS, RANK, ADAPTERS = 40, 512, 264, 300, 16, 3


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def bf(*shape, seed):
    return inputs.gaussian_bf16(shape, seed, std=1.0, device=DEV)


def calls(nz):
    """Each operator that takes scratch memory: a call with its results at hand, those, and how far two calls' may lie apart: the linear
    layer's sums come in any order."""
    x, gate, up = bf(TOKENS, IN, seed=1), bf(OUT, IN, seed=2), bf(OUT, IN, seed=3)
    blobs = [nz.neuzip_compress(w, 7) for w in (gate, up)]
    tokens, grad_out = (torch.arange(600, device=DEV) * 7) % ROWS, bf(600, IN, seed=10)
    ids = (torch.arange(TOKENS, device=DEV) % ADAPTERS).to(torch.int32)
    a, b = bf(ADAPTERS, RANK, IN, seed=4), bf(ADAPTERS, OUT, RANK, seed=5)
    g, u = bf(TOKENS, OUT, seed=6).float(), bf(TOKENS, OUT, seed=7).float()
    h, grad, y = torch.empty_like(g, dtype=torch.bfloat16), torch.empty(ROWS, IN, dtype=torch.bfloat16, device=DEV), torch.empty_like(g)
    gx, gw = torch.empty_like(x), (torch.empty_like(gate), torch.empty_like(up))
    gh = bf(TOKENS, OUT, seed=8)
    xm, sums = x.float().abs(), 2.0 * (IN + RANK + 64) * 2.0 ** -24     # (the classical bound of a float32 sum, for each of the two)
    of_gate, of_up = (2.0 * sums * (xm @ w.float().abs().t()).max().item() for w in (gate, up))
    gm, um = ((x.float() @ w.float().t()).abs().max().item() for w in (gate, up))
    of_h = 1.2 * of_gate * um + of_up * gm + 2.0 ** -7 * gm * um        # (the activation's slope; a rounding to bf16 each)
    low = sum((xm @ a[i].float().abs().t()) @ b[i].float().abs().t() for i in range(ADAPTERS)).max().item()
    return {
        "embedding_grad": (lambda **kw: nz.neuzip_embedding_grad(tokens, grad_out, ROWS, 1.0, grad, **kw), [grad], 0.0),
        "gated_linear": (lambda **kw: nz.neuzip_gated_linear(*blobs, OUT, IN, x, nz.SILU, h, **kw), [h], of_h),
        "gated_backward": (lambda **kw: nz.neuzip_gated_backward(x, gate, up, g, u, gh, nz.SILU, gx, gw, **kw), [gx, *gw], 0.0),
        "linear_adapters": (lambda **kw: nz.neuzip_linear_adapters(blobs[0], OUT, IN, x, a, b, None, ids, None, y, **kw), [y], of_gate + 2.0 * sums * low),
    }


@pytest.mark.parametrize("name", ["embedding_grad", "gated_linear", "gated_backward", "linear_adapters"])
def test_scratch_memory_while_another_thread_captures(nz, name):
    call, results, apart = calls(nz)[name]
    call()
    torch.cuda.synchronize()
    want = [r.clone() for r in results]
    for r in results:
        r.fill_(7)
    side = torch.cuda.Stream()
    count = torch.ones(1000, device=DEV)
    torch.cuda.synchronize()
    failed = []

    def other():
        try:
            call(stream=side)
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
    for r, w in zip(results, want):
        assert (r.float() - w.float()).abs().max().item() <= apart


def test_more_than_a_launch_has_room_for(nz):
    blob = nz.neuzip_compress(bf(ROWS, IN, seed=9), 7)
    room = torch.zeros(64, dtype=torch.int64, device=DEV)
    at = ctypes.c_void_p(room.data_ptr())
    for count in (1 << 27, 1 << 31, 1 << 40, (1 << 64) - 1):
        assert nz._lib.neuzip_embedding(blob.handle, ROWS, IN, at, count, 1.0, at, None) == nz.EUNSUPPORTED
        assert nz._lib.neuzip_embedding_grad(at, max(count, 1 << 31), at, ROWS, IN, 1.0, at, at, 512, None) == nz.EUNSUPPORTED
    torch.cuda.synchronize()
    assert bool((room == 0).all())
