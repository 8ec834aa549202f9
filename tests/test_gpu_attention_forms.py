"""Every form of the attention's kernels at sizes that take it, against float64 on the GPU, within the bound that cache_reference.py derives (-m gpu).
tests/test_attention_forms.py (no GPU) sees to it that each form that the library's rule can choose is taken by a case here.
"""
import math

import pytest
import torch

from cache_reference import E4M3
from test_gpu_cache import DEV, ints, starts_of, tables

pytestmark = pytest.mark.gpu

# heads, group, head_dim, page, window, (new tokens, tokens with them) of each sequence
CASES = {
    "few, eight waves": (2, 4, 128, 64, 0, [(1, 3000), (2, 1), (1, 999), (3, 400)]),
    "few, eight waves, one round": (2, 4, 64, 16, 0, [(1, 700), (1, 64), (3, 65)]),
    "few, four waves": (9, 4, 128, 32, 0, [(1, 100 + 10 * i) for i in range(40)]),
    "few, four waves, split": (12, 3, 64, 128, 0, [(1, 4000 + 50 * i) for i in range(24)]),
    "some": (3, 5, 64, 16, 0, [(130, 700), (77, 77), (0, 40), (300, 301)]),
    "some, window": (2, 4, 128, 64, 100, [(230, 1700), (77, 77)]),
    "some, split": (2, 8, 128, 16, 0, [(33, 3333), (20, 2050)]),
    "many": (8, 4, 128, 64, 0, [(800, 1100), (200, 200), (330, 1000)]),
    "many, short pages": (8, 4, 128, 16, 0, [(800, 1100), (200, 200), (330, 1000)]),
    "many, small heads": (8, 5, 64, 32, 0, [(1600, 1600), (700, 900), (40, 41)]),
    "many, small heads, wide pages": (8, 5, 64, 128, 300, [(1600, 1600), (700, 900), (40, 41)]),
    "many, split": (4, 8, 128, 128, 0, [(1300, 2500), (100, 900)]),
    "many, split, short pages": (4, 3, 128, 32, 0, [(600, 9100), (0, 3000), (300, 4000)]),
    "most": (8, 4, 128, 64, 0, [(3300, 3300), (900, 900)]),
    "most, split": (4, 4, 128, 128, 0, [(500, 9100), (0, 70), (300, 4000)]),
    "most, window": (8, 4, 128, 64, 3111, [(3500, 4200), (1, 1), (700, 900)]),
    "many, small heads, short prompts": (8, 4, 64, 32, 0, [(400, 410), (380, 380), (500, 700), (600, 600)]),
    "many, window": (8, 4, 128, 64, 777, [(1000, 2300), (600, 600)]),
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
    heads, group, dim, page, window, plan = CASES[case]
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


def expected(cache, table, starts, lengths, q, window):
    """(out, bound) as in cache_reference.attend, on the GPU."""
    out, bound = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    page, dim, heads = cache.page_tokens, cache.head_dim, cache.heads
    group, scale = q.shape[1] // heads, dim ** -0.5
    for s, length in enumerate(lengths):
        at = slice(starts[s], starts[s + 1])
        n = starts[s + 1] - starts[s]
        if n == 0 or n > length:
            continue
        to = torch.tensor(table[s][:(length + page - 1) // page], device=DEV)
        position, key = torch.arange(length - n, length, device=DEV)[:, None], torch.arange(length, device=DEV)
        hidden = (key > position) | (key <= position - window if window else False)
        for h in range(heads):
            k = (cache.k.view(torch.uint8)[to, h].view(E4M3).double() * cache.k_scales[to, h].double()[:, None, None]).reshape(-1, dim)[:length]
            v = (cache.v.view(torch.uint8)[to, h].view(E4M3).double() * cache.v_scales[to, h].double()[:, None, None]).transpose(1, 2).reshape(-1, dim)[:length]
            for j in range(h * group, (h + 1) * group):
                query = q[at, j].double()
                p = torch.softmax((query @ k.t() * scale).masked_fill(hidden, -math.inf), dim=1)
                spread = ((query.abs() @ k.abs().t()).masked_fill(hidden, 0).amax(dim=1) * scale)[:, None]
                o, whole = p @ v, p @ v.abs()
                each = 2.0 ** -8 + (2 * (dim + 8) * spread + length / 16 + 300) * 2.0 ** -24
                out[at, j], bound[at, j] = o, each * whole * (1 + 2.0 ** -7) + 2.0 ** -8 * o.abs() + 1e-30
    return out, bound


@pytest.mark.parametrize("case", CASES)
def test_form(nz, case):
    heads, group, dim, page, window, _ = CASES[case]
    cache, table, starts, lengths = made(nz, case, 100)
    q = normal(starts[-1] + 5, heads * group, dim, seed=110).to(torch.bfloat16)
    got = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    sequences = nz.Sequences(ints(starts), ints(lengths), ints(table))
    nz.neuzip_cache_attention(cache, sequences, q, window=window, out=got)
    want, bound = expected(cache, table, starts, lengths, q, window)
    off = ((got.double() - want).abs() - bound)[:starts[-1]]
    assert not bool(torch.isnan(off).any()) and bool((off <= 0).all()), float(off.max())
    assert bool((got[starts[-1]:] == 7.0).all())
    again = nz.neuzip_cache_attention(cache, sequences, q, window=window)
    assert torch.equal(again[:starts[-1]], got[:starts[-1]])


@pytest.mark.parametrize("case", [c for c in CASES if c != "few, eight waves, one round"])
def test_form_with_pages_that_are_not_there_and_nan(nz, case):
    """One page of the first sequence is nowhere, one of its last values NaN: as if the page's tokens had been masked, and NaN for those who see it."""
    heads, group, dim, page, window, _ = CASES[case]
    cache, table, starts, lengths = made(nz, case, 120)
    q = normal(starts[-1], heads * group, dim, seed=130).to(torch.bfloat16)
    sequences = nz.Sequences(ints(starts), ints(lengths), ints(table))
    n, length = starts[1], lengths[0]
    gone = max(0, (length - n - (20 if window else page + 20)) // page)
    low, high = gone * page, min((gone + 1) * page, length)
    hole = [row[:] for row in table]
    hole[0][gone] = -1 if gone % 2 else 1 << 28
    got = nz.neuzip_cache_attention(cache, nz.Sequences(ints(starts), ints(lengths), ints(hole)), q, window=window)
    to = torch.tensor(table[0][:(length + page - 1) // page], device=DEV)
    position, key = torch.arange(length - n, length, device=DEV)[:, None], torch.arange(length, device=DEV)
    hidden = (key > position) | (key <= position - window if window else False) | ((key >= low) & (key < high))
    for h in (0, heads - 1):
        k = (cache.k.view(torch.uint8)[to, h].view(E4M3).double() * cache.k_scales[to, h].double()[:, None, None]).reshape(-1, dim)[:length]
        v = (cache.v.view(torch.uint8)[to, h].view(E4M3).double() * cache.v_scales[to, h].double()[:, None, None]).transpose(1, 2).reshape(-1, dim)[:length]
        p = torch.softmax((q[:n, h * group].double() @ k.t() * dim ** -0.5).masked_fill(hidden, -math.inf), dim=1)
        p = torch.nan_to_num(p)         # (a row that sees nothing: zeros)
        spread = float((q[:n, h * group].double().abs() @ k.abs().t()).max()) * dim ** -0.5
        bound = (2.0 ** -8 + (2 * (dim + 8) * spread + length / 16 + 300) * 2.0 ** -24) * (p @ v.abs()) * (1 + 2.0 ** -7) + 2.0 ** -8 * (p @ v).abs() + 1e-30
        off = (got[:n, h * group].double() - p @ v).abs() - bound
        assert not bool(torch.isnan(off).any()) and bool((off <= 0).all()), float(off.max())
    before = nz.neuzip_cache_attention(cache, sequences, q, window=window)
    poisoned, feature, head = length - (n + 1) // 2, dim - 3, heads - 1
    cache.v.view(torch.uint8)[table[0][poisoned // page], head, feature, poisoned % page] = 0x7F
    got = nz.neuzip_cache_attention(cache, sequences, q, window=window)
    sees = torch.zeros(q.shape[0], dtype=torch.bool, device=DEV)
    sees[:n] = torch.arange(length - n, length, device=DEV) >= poisoned
    if window:
        sees[:n] &= torch.arange(length - n, length, device=DEV) < poisoned + window
    mine = torch.zeros_like(got, dtype=torch.bool)
    mine[:, head * group:, feature] = sees[:, None]
    assert bool(sees.any()) and torch.equal(torch.isnan(got), mine)
    # (the NaN is taken as 0 in the other products' sums: those rows keep their bits)
    assert torch.equal(got[~sees], before[~sees]) and torch.equal(got[sees][..., :feature], before[sees][..., :feature])
