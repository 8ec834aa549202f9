"""Plain statements of the cache of 8-bit keys and values, shared by its tests: which pages tokens go to, what the bytes are, and attention in 64 bits."""
import math

import torch

E4M3 = torch.float8_e4m3fn


def scale_for(most: float) -> float:
    """The least power of two from 2^-100 on by which `most` is at most 448."""
    e = -100
    while most > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Cache:
    """pages x heads of float64 values, the bytes' own (without scale), and the scales."""

    def __init__(self, k, v, k_scales, v_scales):
        self.k = k.cpu().float().double()
        self.v = v.cpu().float().double().transpose(2, 3).contiguous()
        self.k_scales, self.v_scales = k_scales.cpu().double(), v_scales.cpu().double()

    def append(self, starts, lengths, table, k, v, rotary=None):
        """k, v: rows x heads x features (CPU)."""
        pages, heads, page, _ = self.k.shape
        for s in range(len(lengths)):
            rows, length = range(starts[s], starts[s + 1]), lengths[s]
            first = length - len(rows)
            if first < 0 or length > len(table[s]) * page:
                continue
            for number in range(first // page, (length + page - 1) // page if len(rows) else 0):
                to = table[s][number]
                if not 0 <= to < pages:
                    continue
                places = [p for p in range(number * page, (number + 1) * page) if first <= p < length]
                begin = places[0] - number * page
                at = [rows[p - first] for p in places]
                for held, scales, x, turn in ((self.k, self.k_scales, k, rotary), (self.v, self.v_scales, v, None)):
                    x = x[at].float()
                    if turn is not None:
                        x = rotated(x, turn[places])
                    for h in range(heads):
                        some = x[:, h]
                        finite = some[torch.isfinite(some)].abs()
                        scale = scale_for(float(finite.max()) if finite.numel() else 0.0)
                        if begin:
                            scale = max(scale, float(scales[to, h]))
                            held[to, h, :begin] = coded(held[to, h, :begin].float() * (float(scales[to, h]) / scale)).double()
                        scales[to, h] = scale
                        held[to, h, begin:begin + len(places)] = coded(some * (1.0 / scale)).double()


def coded(x):
    """float32 to the nearest value of e4m3; beyond its largest, that."""
    return x.clamp(-448.0, 448.0).to(E4M3).float()


def rotated(x, angles):
    """float32, each product and sum rounded."""
    half = x.shape[-1] // 2
    cos, sin = angles[:, None, :half], angles[:, None, half:]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def attend(cache, starts, lengths, table, q, scale, window=0):
    """(out, bound on what binary32 sums and weights rounded to bf16 may be off, seen) in float64 of a Cache; q: rows x query heads x features
    (CPU).  seen: rows that belong to a sequence.

    The weights p are rounded to bf16, half a step 2^-8 of each: at most 2^-8 sum p |v|.  A score of D products, exact, summed in binary32, is off by
    at most D 2^-24 sum |q k|, a few more roundings of it in the exponent; that much relative to p, and once more in the sum of them; the sums over n keys, in
    steps of 64 over 4 waves and up to 128 splits, by less than (n / 16 + 300) 2^-24.  The result is rounded to bf16."""
    out, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    seen = torch.zeros(q.shape[0], dtype=torch.bool)
    pages, heads, page, dim = cache.k.shape
    group = q.shape[1] // heads
    for s in range(len(lengths)):
        n, length = starts[s + 1] - starts[s], lengths[s]
        seen[starts[s]:starts[s + 1]] = True
        if n <= 0 or n > length or length > len(table[s]) * page:
            continue
        numbers = [table[s][i] for i in range((length + page - 1) // page)]
        there = torch.tensor([0 <= p < pages for p in numbers]).repeat_interleave(page)[:length]
        at = torch.tensor([p if 0 <= p < pages else 0 for p in numbers])
        where = torch.arange(length)
        for i in range(n):
            position = length - n + i
            sees = there & (where <= position)
            if window:
                sees &= where > position - window
            if not bool(sees.any()):
                continue
            for h in range(heads):
                k = (cache.k[at, h] * cache.k_scales[at, h][:, None, None]).reshape(-1, dim)[:length][sees]
                v = (cache.v[at, h] * cache.v_scales[at, h][:, None, None]).reshape(-1, dim)[:length][sees]
                query = q[starts[s] + i, h * group:(h + 1) * group].double()
                score = query @ k.t() * scale
                p = torch.softmax(score, dim=1)
                spread = (query.abs() @ k.abs().t()).max(dim=1).values * scale
                o, whole = p @ v, p @ v.abs()
                each = 2.0 ** -8 + (2 * (dim + 8) * spread + k.shape[0] / 16 + 300) * 2.0 ** -24
                out[starts[s] + i, h * group:(h + 1) * group] = o
                bound[starts[s] + i, h * group:(h + 1) * group] = each[:, None] * whole * (1 + 2.0 ** -7) + 2.0 ** -8 * o.abs() + 1e-30
    return out, bound, seen
