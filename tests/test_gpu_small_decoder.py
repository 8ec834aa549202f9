"""Norms, attention with its cache, gated blocks and logits together, as the small model and the small decoder run them (-m gpu)."""
import math

import pytest
import torch

from paper_2410_20650_amd import inputs
from test_gpu_small_model import held, weights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("tokens", [40, 300])
def test_a_step_with_a_norm_is_the_plain_one(tokens):
    """The model with a norm against its formula in 64 bits, differentiated by torch on the CPU; as near as the model without is (bf16 words all along the
    way: in the mean a few per cent of the step)."""
    from paper_2410_20650_amd.small_model import SmallModel
    model = SmallModel(rows=500, norm=True)
    before, norm_before = weights(model), model.norm.weight.clone()
    g = torch.Generator().manual_seed(3)
    tok = torch.randint(0, 500, (tokens,), generator=g).to(DEV)
    target = inputs.gaussian_bf16((tokens, 128), 21, std=1.0, device=DEV)
    lr = 8.0
    loss = model.training_step(tok, target, lr)
    leaves = [w.double().cpu().requires_grad_() for w in (*before, norm_before)]
    table, gate, up, down, out, weight = leaves
    h = model.embedding.scale * table[tok.cpu()]
    n = h / (h.square().mean(dim=1, keepdim=True) + model.norm.eps).sqrt() * weight
    a, b = n @ gate.t(), n @ up.t()
    y = (h + (a * torch.sigmoid(a) * b) @ down.t()) @ out.t()
    want = 0.5 * ((y - target.double().cpu()) ** 2).sum() / tokens
    want.backward()
    assert abs(loss - float(want.detach())) <= 0.02 * float(want.detach())
    for leaf, old, new in zip(leaves, (*before, norm_before), (*weights(model), model.norm.weight)):
        moved, right = (old.double() - new.double()).cpu(), lr * leaf.grad
        rounding = 2.0 ** -8 if new.dtype == torch.bfloat16 else 2.0 ** -24
        assert float((moved - right).norm()) <= 0.05 * float(right.norm()) + rounding * float(new.double().norm())
        assert bool(((moved - right).abs() <= rounding * new.double().cpu().abs() + 0.1 * right.abs().max()).all())


@pytest.mark.parametrize("counts, lengths", [([1, 1, 1], [5, 64, 200]), ([70, 3], [70, 130])])
def test_the_attention_block_is_its_parts(nz, counts, lengths):
    """CompressedAttention against the same calls one by one, weights decompressed, products in float64: the cache within a step of e4m3, and the output
    within what bf16 queries and e4m3 keys and values (2^-4 of themselves at most) make of it."""
    from paper_2410_20650_amd.layer import CompressedAttention
    width, heads, group, dim, page = 256, 2, 3, 64, 32
    shapes = [(heads * group * dim, width), (heads * dim, width), (heads * dim, width), (width, heads * group * dim)]
    ws = [inputs.gaussian_bf16(s, 900 + i, std=s[1] ** -0.5, device=DEV) for i, s in enumerate(shapes)]
    block = CompressedAttention(*ws, dim, window=90)
    pages = [(n + page - 1) // page for n in lengths]
    at, table = 0, []
    for n in pages:
        table.append(list(range(at, at + n)) + [-1] * (max(pages) - n))
        at += n
    cache = block.new_cache(at, page, DEV)
    space = torch.zeros(heads * group * dim * width, dtype=torch.bfloat16, device=DEV)
    x = [inputs.gaussian_bf16((n, width), 950 + i, std=1.0, device=DEV) for i, n in enumerate(lengths)]
    first = [n - c for n, c in zip(lengths, counts)]
    if any(first):
        starts = torch.tensor([0] + first).cumsum(0).tolist()
        block.forward(torch.cat([t[:n] for t, n in zip(x, first)]), cache, nz.Sequences(ints(starts), ints(first), ints(table)), space)
    starts = torch.tensor([0] + counts).cumsum(0).tolist()
    got = block.forward(torch.cat([t[n:] for t, n in zip(x, first)]), cache, nz.Sequences(ints(starts), ints(lengths), ints(table)), space)
    assert got.dtype == torch.float32 and got.shape == (starts[-1], width)
    wq, wk, wv, wo = (held(p.blob, s).double() for p, s in zip((block.queries, block.keys, block.values, block.out), shapes))
    for s, n in enumerate(lengths):
        k, v = ((x[s].double() @ w.t()).view(n, heads, dim) for w in (wk, wv))
        for h in range(heads):
            bytes_ = cache.k.view(torch.uint8)[table[s][:pages[s]], h].view(torch.float8_e4m3fn).double() * cache.k_scales[table[s][:pages[s]], h].double()[:, None, None]
            there = bytes_.reshape(-1, dim)[:n]
            largest = cache.k_scales[table[s][:pages[s]], h].double().repeat_interleave(page)[:n, None]
            # half a step of a normal value, half a subnormal step, and what the binary32 product may be off; twice where a token's page was rounded anew
            assert bool(((there - k[:, h]).abs() <= 2 * (2.0 ** -4 * k[:, h].abs() + 2.0 ** -10 * largest) + 1e-4).all())
        q = (x[s][first[s]:].double() @ wq.t()).view(counts[s], heads, group, dim)
        position, key = torch.arange(first[s], n, device=DEV)[:, None], torch.arange(n, device=DEV)
        hidden = (key > position) | (key <= position - 90)
        seen = torch.empty(counts[s], heads, group, dim, dtype=torch.float64, device=DEV)
        for h in range(heads):
            for j in range(group):
                p = torch.softmax((q[:, h, j] @ k[:, h].t() * dim ** -0.5).masked_fill(hidden, -math.inf), dim=1)
                seen[:, h, j] = p @ v[:, h]
        want = seen.view(counts[s], -1) @ wo.t()
        assert float((got[starts[s]:starts[s + 1]].double() - want).norm()) <= 2.0 ** -4 * float(want.norm())


def test_tokens_one_by_one_and_at_once(nz):
    """A prompt through the decoder in one call, in parts, and token by token: the same but for bf16's and e4m3's roundings."""
    from paper_2410_20650_amd.small_model import SmallDecoder
    decoder = SmallDecoder(rows=300)
    tokens = torch.randint(0, 300, (90,), generator=torch.Generator().manual_seed(4)).to(DEV)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    answers = []
    for parts in ([90], [64, 20, 6], [1] * 90):
        caches, at, rows = decoder.caches(2), 0, []
        for n in parts:
            at += n
            rows.append(decoder.forward(tokens[at - n:at], caches, nz.Sequences(ints([0, n]), ints([at]), table)))
        answers.append(torch.cat(rows))
    assert bool(torch.isfinite(answers[0]).all())
    for other in answers[1:]:
        assert float((other - answers[0]).norm()) <= 2.0 ** -4 * float(answers[0].norm())


def test_answers(nz):
    from paper_2410_20650_amd.small_model import SmallDecoder
    decoder = SmallDecoder(rows=200, window=50)
    prompts = [torch.arange(n, device=DEV) * 7 % 200 for n in (3, 80, 1)]
    answers = decoder.answer(prompts, 20, presence=1e9, page_tokens=32)
    assert answers.shape == (3, 20) and bool(((answers >= 0) & (answers < 200)).all())
    for row in answers.tolist():
        assert len(set(row)) == 20                  # no token twice: the penalty is more than any logit
    allowed = torch.zeros(7, dtype=torch.int32, device=DEV)
    allowed[1] = 0b1010000                          # tokens 36 and 38
    few = decoder.answer(prompts, 6, allowed=allowed, bias=(torch.tensor([38], device=DEV), torch.tensor([1e6], device=DEV)))
    assert bool((few == 38).all())
    with pytest.raises(ValueError):
        decoder.answer(prompts, 2000)


def test_the_command(capsys):
    from paper_2410_20650_amd import small_model
    small_model.main(["--steps", "2", "--tokens", "100", "--norm", "--answer", "4"])
    assert capsys.readouterr().out.count("answer to") == 3


def test_layers_refuse_what_they_cannot_hold():
    from paper_2410_20650_amd.layer import CompressedAttention
    w = [inputs.gaussian_bf16(s, 980 + i, device=DEV) for i, s in enumerate([(256, 256), (128, 256), (128, 256), (256, 256)])]
    for i, bad in ((0, (192, 256)), (1, (100, 256)), (2, (64, 256)), (3, (256, 128))):
        with pytest.raises(ValueError):
            CompressedAttention(*[inputs.gaussian_bf16(bad, 990, device=DEV) if j == i else t for j, t in enumerate(w)], 64)


def test_no_rows_and_no_prompt(nz):
    from paper_2410_20650_amd.small_model import SmallDecoder
    decoder = SmallDecoder(rows=100, layers=1)
    attention = decoder.layers[0][1]
    nobody = nz.Sequences(ints([0, 0]), ints([0]), ints([[0]]))
    none = torch.empty((0, 256), dtype=torch.bfloat16, device=DEV)
    assert attention.forward(none, attention.new_cache(1, 64, DEV), nobody, decoder.space).shape == (0, 256)
    for prompts in ([], [torch.arange(3, device=DEV), torch.arange(0, device=DEV)]):
        with pytest.raises(ValueError):
            decoder.answer(prompts, 2)
