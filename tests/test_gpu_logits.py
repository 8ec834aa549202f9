"""Penalties, biases and masks on logits, bit for bit against the same operations on the CPU, each rounded to binary32 by itself (-m gpu)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def plain(logits, histories=None, repetition=None, frequency=None, presence=None, biases=None, masks=None, mask_ids=None):
    """On the CPU; histories and biases: a list for each row."""
    out = logits.clone()
    rows, vocab = logits.shape
    for r in range(rows):
        x = out[r]
        if histories is not None:
            here = [t for t in histories[r] if 0 <= t < vocab]
            count = torch.bincount(torch.tensor(here, dtype=torch.int64), minlength=vocab).float()
            rep = repetition[r] if repetition is not None else torch.tensor(1.0)
            x = torch.where(count > 0, torch.where(x > 0, x / rep, x * rep), x)
            if frequency is not None:
                x = torch.where(count > 0, x - frequency[r] * count, x)
            if presence is not None:
                x = torch.where(count > 0, x - presence[r], x)
        if biases is not None:
            for token, value in dict(biases[r]).items():
                if 0 <= token < vocab:
                    x[token] = x[token] + torch.tensor(value)
        if masks is not None and 0 <= int(mask_ids[r]) < masks.shape[0]:
            bits = (masks[int(mask_ids[r])].long()[:, None] >> torch.arange(32)) & 1
            x = torch.where(bits.reshape(-1)[:vocab] == 1, x, torch.tensor(-math.inf))
        out[r] = x
    return out


def ragged(lists, dtype):
    starts = [0]
    for one in lists:
        starts.append(starts[-1] + len(one))
    return (torch.tensor([v for one in lists for v in one], dtype=dtype, device=DEV), torch.tensor(starts, dtype=torch.int32, device=DEV))


def case(rows, vocab, seed, history, bias):
    g = torch.Generator()
    g.manual_seed(seed)
    logits = torch.randn(rows, vocab, generator=g) * 3
    histories = [[int(t) for t in torch.randint(-2, vocab + 2, (int(history * (r + 1) / rows),), generator=g)] for r in range(rows)]
    for h in histories:
        h.extend(h[:len(h) // 2])           # tokens that occur several times
    biases = [[(int(t), float(v)) for t, v in zip(torch.randint(-1, vocab + 1, (bias + r,), generator=g), torch.randn(bias + r, generator=g))] for r in range(rows)]
    for b in biases:
        if len(b) > 1:
            b.append((b[0][0], 0.25))       # a token that is named twice
    penalties = [1 + torch.rand(rows, generator=g) * 0.5 for _ in range(3)]
    masks = torch.randint(-2 ** 31, 2 ** 31, (3, (vocab + 31) // 32), generator=g).to(torch.int32)
    masks[2] = 0                            # allows nothing
    ids = torch.tensor([(-1, 0, 1, 2, 3)[r % 5] for r in range(rows)], dtype=torch.int32)
    return logits, histories, penalties, biases, masks, ids


@pytest.mark.parametrize("history, bias", [(0, 0), (1, 1), (40, 5), (3000, 300)])
@pytest.mark.parametrize("rows, vocab", [(1, 1), (2, 31), (5, 1000), (3, 1024), (7, 4097), (1, 128256), (6, 50257), (70, 2049), (22, 50257), (9, 128256)])
def test_everything(nz, rows, vocab, history, bias):
    logits, histories, (repetition, frequency, presence), biases, masks, ids = case(rows, vocab, 3, history, bias)
    tokens, starts = ragged(histories, torch.int64)
    named, bias_starts = ragged([[t for t, _ in b] for b in biases], torch.int64)
    values, _ = ragged([[v for _, v in b] for b in biases], torch.float32)
    want = plain(logits, histories, repetition, frequency, presence, biases, masks, ids)
    on = [t.to(DEV) for t in (repetition, frequency, presence)]
    mine = logits.to(DEV)
    got = nz.neuzip_logits(mine, tokens, starts, *on, named, values, bias_starts, masks.to(DEV), ids.to(DEV))
    assert torch.equal(got.cpu(), want) and torch.equal(mine.cpu(), logits)
    assert nz.neuzip_logits(mine, tokens, starts, *on, named, values, bias_starts, masks.to(DEV), ids.to(DEV), mine) is mine
    assert torch.equal(mine.cpu(), want)


def test_one_by_one(nz):
    logits, histories, (repetition, frequency, presence), biases, masks, ids = case(6, 5003, 4, 100, 10)
    tokens, starts = ragged(histories, torch.int64)
    named, bias_starts = ragged([[t for t, _ in b] for b in biases], torch.int64)
    values, _ = ragged([[v for _, v in b] for b in biases], torch.float32)
    on = logits.to(DEV)
    assert torch.equal(nz.neuzip_logits(on).cpu(), logits)
    assert torch.equal(nz.neuzip_logits(on, tokens, starts).cpu(), logits)
    assert torch.equal(nz.neuzip_logits(on, tokens, starts, repetition.to(DEV)).cpu(), plain(logits, histories, repetition))
    assert torch.equal(nz.neuzip_logits(on, tokens, starts, frequency=frequency.to(DEV)).cpu(), plain(logits, histories, None, frequency))
    assert torch.equal(nz.neuzip_logits(on, tokens, starts, presence=presence.to(DEV)).cpu(), plain(logits, histories, None, None, presence))
    assert torch.equal(nz.neuzip_logits(on, bias=named, bias_values=values, bias_starts=bias_starts).cpu(), plain(logits, biases=biases))
    assert torch.equal(nz.neuzip_logits(on, masks=masks.to(DEV), mask_ids=ids.to(DEV)).cpu(), plain(logits, masks=masks, mask_ids=ids))


def test_infinities_and_nan(nz):
    """A masked logit is -infinity whatever it was; others stay what the operations make of them."""
    logits = torch.tensor([[math.nan, math.inf, -math.inf, -3.4e38, 1.0, -0.0, math.nan, 2.0]]).repeat(2, 1)
    histories = [[1, 2, 3, 4, 5, 6], [0, 0, 7]]
    masks = torch.tensor([[0b10111110]], dtype=torch.int32)
    ids = torch.zeros(2, dtype=torch.int32)
    repetition, presence = torch.tensor([2.0, 2.0]), torch.tensor([0.5, 0.5])
    tokens, starts = ragged(histories, torch.int64)
    got = nz.neuzip_logits(logits.to(DEV), tokens, starts, repetition.to(DEV), None, presence.to(DEV), masks=masks.to(DEV), mask_ids=ids.to(DEV)).cpu()
    want = plain(logits, histories, repetition, None, presence, masks=masks, mask_ids=ids)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got, nan=5.0), torch.nan_to_num(want, nan=5.0))
    assert bool((got[:, [0, 6]] == -math.inf).all())


def test_starts_beyond_what_is_there(nz):
    """Are taken as the end of what is there; rows without entries are rows without history."""
    logits = torch.zeros(3, 50)
    tokens = torch.tensor([3, 4, 5], dtype=torch.int64, device=DEV)
    starts = torch.tensor([-5, 1, 1, 1 << 30], dtype=torch.int32, device=DEV)
    got = nz.neuzip_logits(logits.to(DEV), tokens, starts, presence=torch.ones(3, device=DEV)).cpu()
    assert got.nonzero().tolist() == [[0, 3], [2, 4], [2, 5]] and bool((got[got != 0] == -1).all())


def test_no_rows(nz):
    assert nz.neuzip_logits(torch.empty(0, 100, device=DEV)).shape == (0, 100)
