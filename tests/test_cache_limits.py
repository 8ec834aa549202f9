"""Calls on the cache that are more than a launch holds, as the header has them: refused before any device work."""
import pytest

from paper_2410_20650_amd import binding as nz
from test_more_operator_arguments import SOME, append, attention, c_cache, c_sequences


@pytest.mark.parametrize("heads, group, rows", [(256, 1, 1 << 15), (1 << 13, 1, 1 << 10), (32, 4, 1 << 18)])
def test_single_tokens_of_many_sequences(heads, group, rows):
    """A workgroup for each of them and head, 2^23 in all: refused though rows * q_heads is below 2^27."""
    q_heads = heads * group
    assert rows * heads == 1 << 23 and rows * q_heads < 1 << 27
    assert attention(c_cache(heads=heads), c_sequences(count=rows), q_row=q_heads * 64, q_heads=q_heads, rows=rows) == nz.EUNSUPPORTED


@pytest.mark.parametrize("page, heads, count, rows, queries", [(16, 64, 1 << 16, 1, False), (16, 1 << 6, 4, 1 << 21, False), (64, 2, 4, 1 << 24, True)])
def test_appends(page, heads, count, rows, queries):
    """(rows / page_tokens + 2 count) * 2 heads workgroups, and one for each row with queries: 2^24 of them."""
    wgs = (rows // page + 2 * count) * 2 * heads + (rows if queries else 0)
    assert wgs >= 1 << 24
    q = dict(q=SOME, q_out=SOME, q_heads=2, q_row=128) if queries else {}
    assert append(c_cache(heads=heads, page_tokens=page), c_sequences(count=count), k_row=heads * 64, v_row=heads * 64, rows=rows, **q) == nz.EUNSUPPORTED


def test_heads():
    assert append(c_cache(heads=1 << 16), k_row=1 << 22, v_row=1 << 22, rows=3) == nz.EUNSUPPORTED
