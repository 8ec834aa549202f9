"""Caches and tensors whose offsets pass 32 bits (-m gpu): the same content in a cache's first pages and in its last ones, the last rows of tensors of more than 2^32
elements by themselves.  (Some 30 GB of the device's memory at a time.)
"""
import pytest
import torch

from test_gpu_cache import ints, tables
from test_gpu_attention_forms import expected

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF = torch.bfloat16
MANY = 1 << 32


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    yield binding
    torch.cuda.empty_cache()


def normal(*shape, seed, dtype=BF):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)


def test_pages_behind_32_bits(nz):
    """Every form of the attention's kernels (one token, 130, 1400, 4200 of a sequence) on either content."""
    heads, group, page, dim, pages, length = 8, 4, 64, 128, 70000, 4200
    assert pages * heads * page * dim > MANY and (pages - 100) * heads * page * dim > MANY
    cache = nz.KeyValueCache.empty(pages, heads, dim, page)
    need = (length + page - 1) // page
    places = {"first": list(range(need)), "last": [pages - 1 - i for i in range(need)]}
    k, v = normal(length, heads, dim, seed=1), normal(length, heads, dim, seed=2)
    q = normal(length, heads * group, dim, seed=3)
    outs = {}
    for name, place in places.items():
        for begin, end in ((0, 2900), (2900, length)):    # (the page between them twice)
            nz.neuzip_cache_append(cache, nz.Sequences(ints([0, end - begin]), ints([end]), ints([place])), k[begin:end], v[begin:end])
        outs[name] = [nz.neuzip_cache_attention(cache, nz.Sequences(ints([0, n]), ints([length]), ints([place])), q[length - n:]) for n in (1, 130, 1400, length)]
    first, last = (torch.tensor(places[name], device=DEV) for name in ("first", "last"))
    filled = torch.arange(need * page, device=DEV) < length
    for held in (cache.k.view(torch.uint8).transpose(2, 3), cache.v.view(torch.uint8)):
        low, high = (torch.stack([held[i] for i in at.tolist()]).permute(1, 2, 0, 3).reshape(heads, dim, -1)[..., filled] for at in (first, last))
        assert bool((low != 0).any()) and torch.equal(low, high)
    for held in (cache.k_scales, cache.v_scales):
        assert torch.equal(held[first], held[last])
    for low, high in zip(outs["first"], outs["last"]):
        assert bool((low != 0).any()) and torch.equal(low, high)


def test_rows_behind_32_bits(nz):
    """A prompt of over a million tokens with a window: its last rows against 64 bits."""
    heads, group, page, dim, rows, window = 2, 16, 128, 128, 1 << 20, 40
    rows += 77
    assert rows * heads * group * dim > MANY
    table = tables([rows], page, (rows + page - 1) // page, seed=4)
    cache = nz.KeyValueCache.empty(len(table[0]), heads, dim, page)
    sequences = nz.Sequences(ints([0, rows]), ints([rows]), ints(table))
    q = normal(rows, heads * group, dim, seed=5)
    turned = nz.neuzip_cache_append(cache, sequences, normal(rows, heads, dim, seed=6), normal(rows, heads, dim, seed=7), q)
    assert torch.equal(turned[-300:], q[-300:]) and torch.equal(turned[:300], q[:300])
    del q
    got = nz.neuzip_cache_attention(cache, sequences, turned, window=window)
    n, pages = 200, 4       # the last tokens, as if the last pages were the sequence
    length = rows - (len(table[0]) - pages) * page
    want, bound = expected(cache, [table[0][-pages:]], [0, n], [length], turned[-n:], window)
    off = (got[-n:].double() - want).abs() - bound
    assert not bool(torch.isnan(off).any()) and bool((off <= 0).all()), float(off.max())


def test_norms_of_many_rows(nz):
    tokens, width, eps = (1 << 20) + 5, 4096, 1e-5
    assert tokens * width > MANY
    total, weight = normal(tokens, width, seed=8), normal(width, seed=9, dtype=torch.float32)
    y = nz.neuzip_norm(total, weight, eps)
    assert torch.equal(y[-9:], nz.neuzip_norm(total[-9:], weight, eps)) and torch.equal(y[:9], nz.neuzip_norm(total[:9], weight, eps))
    grad_x, _ = nz.neuzip_norm_backward(total, weight, y, eps, grad_weight=False)       # (y as its own gradient)
    for part in (slice(-9, None), slice(9)):
        assert torch.equal(grad_x[part], nz.neuzip_norm_backward(total[part], weight, y[part], eps, grad_weight=False)[0])


def test_logits_of_many_rows(nz):
    rows, vocab = 34000, 128256
    assert rows * vocab > MANY
    logits = normal(rows, vocab, seed=10, dtype=torch.float32)
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    history = torch.randint(0, vocab, (rows * 20,), generator=g, device=DEV)
    starts = torch.arange(rows + 1, dtype=torch.int32, device=DEV) * 20
    repetition = torch.full((rows,), 1.5, device=DEV)
    last = logits[-3:].clone()
    want = nz.neuzip_logits(last, history[-60:], ints([0, 20, 40, 60]), repetition[-3:])
    got = nz.neuzip_logits(logits, history, starts, repetition, out=logits)
    assert torch.equal(got[-3:], want) and not torch.equal(want, last)
