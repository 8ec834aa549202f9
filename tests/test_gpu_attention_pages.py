"""The attention's kernels that test_gpu_attention_forms.py has no case for, against float64 on the GPU (-m gpu).  Each form (rows and waves to a workgroup, head_dim) is
compiled apart for steps that lie in one page and for steps of several pages, which look pages up and address them in ways of their own; its keys may be split or
not, and what joins few splits is not what joins many.  tests/test_attention_pages.py (no GPU) sees to it that the cases of the two files take every
combination that the library's rule can choose.

Bound, for n keys.  The weights p are rounded to bf16, half a step 2^-8 of each: at most 2^-8 sum p |v|.  A score of D products, exact, summed in binary32, is off by
at most D 2^-24 sum |q k|, with a few more roundings of it in the exponent: that much relative to p, and once more in the sum of them.  The sum of the products and that
of the weights have, in whatever order, at most n additions one behind the other, each half a step 2^-24 of at most the sum of the terms' sizes; and between steps of 64
keys a multiplication by what the maximum grew.  With the joins of waves and splits, some 300 more: (2 n + n / 16 + 300) 2^-24.  The result is rounded to bf16.
"""
import math

import pytest
import torch

from cache_reference import E4M3
from test_gpu_cache import ints, starts_of, tables

pytestmark = pytest.mark.gpu

DEV = "cuda:0"

# heads, group, head_dim, page, window, (new tokens, tokens with them) of each sequence
PADDING = 2     # rows behind the last sequence's
CASES = {
    # 16 rows, eight waves
    "few, 8": (2, 4, 64, 64, 0, [(1, 900), (3, 130), (1, 64), (2, 63)]),
    "few, 8, 128": (1, 8, 128, 128, 0, [(1, 1000), (1, 129)]),
    "few, 8, short pages": (3, 5, 128, 16, 0, [(1, 700), (2, 65), (0, 9), (1, 1)]),
    "few, 8, split": (2, 4, 64, 128, 0, [(1, 5000), (2, 300), (1, 2049)]),
    "few, 8, split, short pages": (2, 4, 64, 16, 0, [(1, 5000), (2, 300), (1, 2049)]),
    "few, 8, split, short pages, 128": (2, 3, 128, 32, 2500, [(1, 4000), (3, 3000)]),
    "few, 8, split far": (1, 4, 64, 64, 0, [(1, 20011)]),
    "few, 8, split far, short pages": (1, 4, 64, 32, 0, [(2, 20011)]),
    "few, 8, split far, 128": (1, 4, 128, 64, 0, [(1, 12001)]),
    "few, 8, split far, short pages, 128": (2, 4, 128, 16, 0, [(1, 12001)]),
    # 16 rows, four waves
    "few, 4": (9, 2, 64, 64, 0, [(1, 50 + 21 * i) for i in range(40)]),
    "few, 4, short pages": (9, 4, 64, 16, 0, [(1, 50 + 21 * i) for i in range(40)]),
    "few, 4, 128": (9, 4, 128, 64, 0, [(1, 50 + 21 * i) for i in range(40)]),
    "few, 4, 128, 70 sequences": (8, 4, 128, 64, 0, [(1, 1 + 13 * i) for i in range(70)]),
    "few, 4, split, short pages": (12, 3, 64, 32, 0, [(1, 1100 + 30 * i) for i in range(24)]),
    "few, 4, split, 128": (8, 4, 128, 64, 0, [(1, 300 + 60 * i) for i in range(48)]),
    "few, 4, split, short pages, 128": (8, 4, 128, 16, 1500, [(1, 300 + 60 * i) for i in range(48)]),
    # 32 rows
    "some": (3, 5, 64, 64, 0, [(130, 400), (77, 77), (0, 40), (300, 301)]),
    "some, 128 sequences": (2, 4, 64, 128, 0, [(9, 9 + i) for i in range(128)]),
    "some, short pages, 128": (2, 4, 128, 16, 0, [(130, 400), (77, 77), (0, 40), (200, 201)]),
    "some, split": (2, 8, 64, 64, 0, [(33, 3333), (20, 2050)]),
    "some, split, short pages": (2, 8, 64, 16, 0, [(33, 3333), (20, 2050)]),
    "some, split, 128": (2, 8, 128, 64, 0, [(33, 3333), (20, 2050)]),
    "some, group of 17": (1, 17, 128, 128, 0, [(1, 1000), (1, 2900)]),
    "some, split far": (1, 4, 64, 128, 0, [(20, 12001)]),
    "some, split far, short pages": (1, 4, 64, 32, 0, [(20, 12001)]),
    "some, split far, 128": (1, 4, 128, 64, 0, [(20, 8001)]),
    "some, split far, short pages, 128": (1, 4, 128, 16, 0, [(20, 8001)]),
    # 128 and 256 rows
    "many, split far": (3, 1, 128, 64, 0, [(2500, 9800)]),
    "many, split far, short pages": (4, 4, 128, 16, 0, [(360, 13000)]),
    "many, 70 sequences": (8, 4, 128, 32, 0, [(40 + i % 7, 60 + i) for i in range(70)]),
    "most, split far": (4, 4, 128, 64, 0, [(360, 13000)]),
}


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def normal(*shape, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV) * std


def made(nz, case, seed):
    """(cache, table, starts, lengths): sequences of that content, the rest NaN."""
    heads, _, dim, page, _, plan = CASES[case]
    lengths = [length for _, length in plan]
    pages = sum((n + page - 1) // page for n in lengths) + 2
    table = tables(lengths, page, pages, seed, width=max((n + page - 1) // page for n in lengths) + 1)
    nan = torch.full((pages, heads, page, dim), 0x7F, dtype=torch.uint8, device=DEV)
    cache = nz.KeyValueCache(nan.view(E4M3), nan.transpose(2, 3).contiguous().view(E4M3),
                             *(torch.full((pages, heads), math.nan, device=DEV) for _ in range(2)))
    starts = starts_of(lengths)
    k = normal(starts[-1], heads, dim, seed=seed + 1) * torch.exp(normal(1, heads, dim, seed=seed + 2, std=0.5))
    nz.neuzip_cache_append(cache, nz.Sequences(ints(starts), ints(lengths), ints(table)), k, normal(starts[-1], heads, dim, seed=seed + 3))
    return cache, table, starts_of([n for n, _ in plan]), lengths


def expected(cache, table, starts, lengths, q, window, only=None):
    """(out, bound) of the rows of the sequences, or of those in `only`; what no token was put to and pages that are not there are seen by nobody."""
    out, bound = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    pages, heads, page, dim = cache.k.shape
    group, scale = q.shape[1] // heads, dim ** -0.5
    for s, length in enumerate(lengths):
        n, at = starts[s + 1] - starts[s], slice(starts[s], starts[s + 1])
        if n == 0 or n > length or (only is not None and s not in only):
            continue
        numbers = table[s][:(length + page - 1) // page]
        to = torch.tensor([p if 0 <= p < pages else 0 for p in numbers], device=DEV)
        there = torch.tensor([0 <= p < pages for p in numbers], device=DEV).repeat_interleave(page)[:length]
        position, key = torch.arange(length - n, length, device=DEV)[:, None], torch.arange(length, device=DEV)
        hidden = (key > position) | ~there
        if window:
            hidden |= key <= position - window
        hidden = hidden.repeat_interleave(group, dim=0)     # rows: token by token, head by head
        for h in range(heads):
            k = (cache.k.view(torch.uint8)[to, h].view(E4M3).double() * cache.k_scales[to, h].double()[:, None, None]).reshape(-1, dim)[:length]
            v = (cache.v.view(torch.uint8)[to, h].view(E4M3).double() * cache.v_scales[to, h].double()[:, None, None]).transpose(1, 2).reshape(-1, dim)[:length]
            k, v = k.masked_fill(~there[:, None], 0), v.masked_fill(~there[:, None], 0)     # (what the page read instead holds is anything)
            query = q[at, h * group:(h + 1) * group].double().reshape(n * group, dim)
            p = torch.nan_to_num(torch.softmax((query @ k.t() * scale).masked_fill(hidden, -math.inf), dim=1))      # (a row that sees nothing: zeros)
            spread = ((query.abs() @ k.abs().t()).masked_fill(hidden, 0).amax(dim=1) * scale)[:, None]
            o, whole = p @ v, p @ v.abs()
            each = 2.0 ** -8 + (2 * (dim + 8) * spread + 2 * length + length / 16 + 300) * 2.0 ** -24
            out[at, h * group:(h + 1) * group] = o.view(n, group, dim)
            bound[at, h * group:(h + 1) * group] = (each * whole * (1 + 2.0 ** -7) + 2.0 ** -8 * o.abs() + 1e-30).view(n, group, dim)
    return out, bound


def within(got, want, bound):
    off = (got.double() - want).abs() - bound
    assert not bool(torch.isnan(off).any()) and bool((off <= 0).all()), float(off.max())


@pytest.mark.parametrize("case", CASES)
def test_form(nz, case):
    heads, group, dim, page, window, _ = CASES[case]
    cache, table, starts, lengths = made(nz, case, 200)
    q = normal(starts[-1] + PADDING, heads * group, dim, seed=210).to(torch.bfloat16)
    got = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    sequences = nz.Sequences(ints(starts), ints(lengths), ints(table))
    nz.neuzip_cache_attention(cache, sequences, q, window=window, out=got)
    want, bound = expected(cache, table, starts, lengths, q, window)
    within(got[:starts[-1]], want[:starts[-1]], bound[:starts[-1]])
    assert bool((got[starts[-1]:] == 7.0).all())
    for _ in range(3):      # the same bits
        again = nz.neuzip_cache_attention(cache, sequences, q, window=window)
        assert torch.equal(again[:starts[-1]], got[:starts[-1]])


@pytest.mark.parametrize("case", CASES)
def test_form_with_pages_that_are_not_there_and_nan(nz, case):
    """A page of the first sequence is nowhere: as if its tokens had been masked.  One of its last values, then one of its last keys, is NaN: so is what the rows that
    see it give, and all else keeps its bits."""
    heads, group, dim, page, window, _ = CASES[case]
    cache, table, starts, lengths = made(nz, case, 220)
    q = normal(starts[-1], heads * group, dim, seed=230).to(torch.bfloat16)
    sequences = nz.Sequences(ints(starts), ints(lengths), ints(table))
    n, length = starts[1], lengths[0]
    before = nz.neuzip_cache_attention(cache, sequences, q, window=window)
    gone = max(0, (length - n - (20 if window else page + 20)) // page)
    hole = [row[:] for row in table]
    hole[0][gone] = -1 if gone % 2 else 1 << 28
    got = nz.neuzip_cache_attention(cache, nz.Sequences(ints(starts), ints(lengths), ints(hole)), q, window=window)
    want, bound = expected(cache, hole, starts, lengths, q, window, only=[0])
    within(got[:n], want[:n], bound[:n])
    assert not torch.equal(got[:n], before[:n]) and torch.equal(got[n:], before[n:])
    poisoned, feature, head = length - (n + 1) // 2, dim - 3, heads - 1
    position = torch.arange(length - n, length, device=DEV)
    sees = torch.zeros(q.shape[0], dtype=torch.bool, device=DEV)
    sees[:n] = position >= poisoned
    if window:
        sees[:n] &= position < poisoned + window
    assert bool(sees.any())
    to, slot = table[0][poisoned // page], poisoned % page
    for held, at in ((cache.v, (to, head, feature, slot)), (cache.k, (to, head, slot, feature))):
        bytes_ = held.view(torch.uint8)
        kept = bytes_[at].clone()
        bytes_[at] = 0x7F
        got = nz.neuzip_cache_attention(cache, sequences, q, window=window)
        bytes_[at] = kept
        mine = torch.zeros_like(got, dtype=torch.bool)
        if held is cache.v:
            mine[:, head * group:, feature] = sees[:, None]
        else:
            mine[:, head * group:] = sees[:, None, None]
        assert torch.equal(torch.isnan(got), mine)
        if held is cache.v:     # (the NaN is taken as 0 in the other products' sums: those rows keep their bits)
            assert torch.equal(got[~sees], before[~sees]) and torch.equal(got[sees][..., :feature], before[sees][..., :feature])
        else:
            assert torch.equal(got[~mine], before[~mine])
    assert torch.equal(nz.neuzip_cache_attention(cache, sequences, q, window=window), before)
