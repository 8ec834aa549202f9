"""Numbers that the library takes in 32 bits: ctypes cuts off what is beyond them, so that 2^32 + 3 rows would be taken for 3 and the others left as they are.  The binding
refuses them.  No GPU: stand-ins for tensors, and nothing reaches the library.
"""
import ctypes

import pytest

from paper_2410_20650_amd import binding as nz
from test_more_operator_arguments import F32, I32, SEQUENCES, Stub, called, reached, sequences  # noqa: F401 (a fixture)

BEYOND = [1 << 32, (1 << 32) + 3]


def test_they_are_cut_off():
    assert ctypes.c_uint32(BEYOND[1]).value == 3


@pytest.mark.parametrize("many", BEYOND)
def test_rows_and_masks_of_logits(called, many):  # noqa: F811
    x = Stub((many, 1), F32)
    with pytest.raises(ValueError):
        nz.neuzip_logits(x)
    with pytest.raises(ValueError):
        nz.neuzip_logits(x, out=x)
    with pytest.raises(ValueError):
        nz.neuzip_logits(Stub((2, 32), F32), masks=Stub((many, 1), I32), mask_ids=Stub((2,), I32), out=Stub((2, 32), F32))
    assert reached(called) == []


@pytest.mark.parametrize("many", BEYOND)
def test_sequences_and_their_pages(called, many):  # noqa: F811
    with pytest.raises(ValueError):
        sequences(Stub((many + 1,), I32), Stub((many,), I32), Stub((many, 1), I32))
    with pytest.raises(ValueError):
        sequences(table=Stub((SEQUENCES, many), I32))


@pytest.mark.parametrize("most", [(1 << 32) - 1])
def test_numbers_of_32_bits_reach_the_library(called, most):  # noqa: F811
    nz.neuzip_logits(Stub((most, 1), F32), out=Stub((most, 1), F32))
    assert reached(called) == ["neuzip_logits"]     # (which refuses them)
    assert sequences(Stub((most + 1,), I32), Stub((most,), I32), Stub((most, 1), I32))._struct.count == most
