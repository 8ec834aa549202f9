"""Shapes of the operators' tensors: as many elements in another order are refused by the binding, dimensions taken together or
apart are not.  No GPU: stand-ins for the tensors, and nothing reaches the library.
"""
import pytest
import torch

from paper_2410_20650_amd import binding as nz
from test_operator_arguments import (ADAPTERS, BLOB, F32, I32, I64, IN, OUT, RANK, ROWS, SCRATCH, TOKENS, Stub, adapters, called, embedding,
                                     embedding_grad, gated_backward, gated_forward, gated_linear)

BF = torch.bfloat16


def up(w_up):
    nz.neuzip_gated_forward(Stub((TOKENS, IN)), Stub((OUT, IN)), w_up, nz.SILU, Stub((TOKENS, OUT)))


def kept_up(up):
    sums = Stub((TOKENS, OUT), F32)
    nz.neuzip_gated_backward(Stub((TOKENS, IN)), Stub((OUT, IN)), Stub((OUT, IN)), sums, up, Stub((TOKENS, OUT)), nz.SILU, Stub((TOKENS, IN)), False, SCRATCH)


def pair(which):
    def call(t):
        two = [Stub((OUT, IN)), Stub((OUT, IN))]
        two[which] = t
        gated_backward(grad_weights=tuple(two))
    return call


def keep(which):
    def call(t):
        two = [Stub((TOKENS, OUT), F32), Stub((TOKENS, OUT), F32)]
        two[which] = t
        gated_forward(keep=tuple(two))
    return call


def named(call, name):
    return lambda t: call(**{name: t})


# a call with one tensor of it at hand, that tensor's shape and type
TENSORS = {
    "embedding out": (named(embedding, "out"), (TOKENS, IN), BF),
    "embedding_grad grad": (named(embedding_grad, "grad"), (ROWS, IN), BF),
    "gated_linear x": (named(gated_linear, "x"), (TOKENS, IN), BF),
    "gated_linear h": (named(gated_linear, "h"), (TOKENS, OUT), BF),
    "gated_forward x": (named(gated_forward, "x"), (TOKENS, IN), BF),
    "gated_forward w_up": (up, (OUT, IN), BF),
    "gated_forward h": (named(gated_forward, "h"), (TOKENS, OUT), BF),
    "gated_forward gate": (keep(0), (TOKENS, OUT), F32),
    "gated_forward up": (keep(1), (TOKENS, OUT), F32),
    "gated_backward x": (named(gated_backward, "x"), (TOKENS, IN), BF),
    "gated_backward gate": (named(gated_backward, "gate"), (TOKENS, OUT), F32),
    "gated_backward up": (kept_up, (TOKENS, OUT), F32),
    "gated_backward grad_h": (named(gated_backward, "grad_h"), (TOKENS, OUT), BF),
    "gated_backward grad_x": (named(gated_backward, "grad_x"), (TOKENS, IN), BF),
    "gated_backward grad_w_gate": (pair(0), (OUT, IN), BF),
    "gated_backward grad_w_up": (pair(1), (OUT, IN), BF),
    "adapters x": (named(adapters, "x"), (TOKENS, IN), BF),
    "adapters b": (named(adapters, "b"), (ADAPTERS, OUT, RANK), BF),
    "adapters y": (named(adapters, "y"), (TOKENS, OUT), F32),
}


def of_the_library(called):
    return [n for n in called if not n.endswith("_scratch_bytes")]


@pytest.mark.parametrize("name", TENSORS)
def test_another_order_is_refused(called, name):
    call, shape, dtype = TENSORS[name]
    *first, n, m = shape
    others = [(*first, m, n), (*first, n // 2, 2 * m), (1, *first, m, n), (*first, m, 1, n)]
    if first:
        others += [(n, *first, m), (m, n, *first), (n, m * first[0])]
    for other in others:
        stub = Stub(other, dtype)
        if stub.numel() != Stub(shape).numel():     # (an odd number halved)
            continue
        with pytest.raises(ValueError):
            call(stub)
    assert of_the_library(called) == []


@pytest.mark.parametrize("name", TENSORS)
def test_the_same_order_is_taken(called, name):
    call, shape, dtype = TENSORS[name]
    *first, n, m = shape
    flat = Stub(shape).numel()
    for same in (shape, (flat,), (1, *shape), (flat // m, m), (1, 1, *shape), (*shape[:-1], m // 2, 2), (*shape[:-2], n, 1, m),
                 (*first, n * m)):
        call(Stub(same, dtype))
    assert len(of_the_library(called)) == 8


def test_numbers_of_tokens_may_have_any_shape(called):
    nz.neuzip_embedding(BLOB, ROWS, IN, Stub((2, TOKENS), I64), 1.0, Stub((2, TOKENS, IN)))
    nz.neuzip_embedding_grad(Stub((2, 3), I64), Stub((2, 3, IN)), ROWS, 1.0, Stub((ROWS * IN,)), SCRATCH)
    nz.neuzip_embedding_grad(Stub((2, 3), I64), Stub((6, IN)), ROWS, 1.0, Stub((ROWS, IN)), SCRATCH)
    adapters(x=Stub((1, TOKENS, IN)), ids=Stub((1, TOKENS), I32), y=Stub((TOKENS, 1, OUT), F32))
    assert of_the_library(called) == ["neuzip_embedding", "neuzip_embedding_grad", "neuzip_embedding_grad", "neuzip_linear_adapters"]
