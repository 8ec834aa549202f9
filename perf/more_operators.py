"""What a compressed model does between its linear layers when it answers, and the sizes a program meets it at.

  norm         the residual's addition and the root-mean-square norm behind it: the next layers' input (bf16) and the stream
  norm_train   the same with its backward pass: the gradients of the stream and of the norm's weight
  append       the keys and values of new tokens rotated to their positions and put into a cache of 8-bit values with a scale for each
               page of tokens and head; the queries rotated and rounded
  attend       attention of the new tokens' queries over that cache, causal, with or without a window
  logits       penalties for tokens that were there, biases, and the mask of a grammar, on the output projection's result

The widths and heads are those of the Llama-3 models that paper_2410_20650_amd/inputs.py lists (4096 wide, 32 query heads on 8 of 128 for keys
and values, 128256 tokens), and generic ones around them.  The plain forms work on the same cache, in binary32.
"""
import math

import torch

own = False

DEV = "cuda"
E4M3 = torch.float8_e4m3fn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def _norm(name, do, tokens, width, x="f32", stream="bf16"):
    c = {"do": do, "tokens": tokens, "width": width, "x": x, "stream": stream}
    return dict(c, name=name) if name else c


def _cached(name, do, sequences, new, longest, heads, group, dim, page=64, window=0, x="f32"):
    """sequences of up to `longest` tokens, the last `new` (or fewer) of them this call's."""
    c = {"do": do, "sequences": sequences, "new": new, "longest": longest, "heads": heads, "group": group, "dim": dim, "page": page}
    c.update({"x": x} if do == "append" else {"window": window})
    return dict(c, name=name) if name else c


def _logits(name, rows, vocab, history, biases, masks):
    c = {"do": "logits", "rows": rows, "vocab": vocab, "history": history, "biases": biases, "masks": masks}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token between two layers: the projection's float32 result onto the bf16 stream
        _norm("norm_1_token", "norm", 1, 4096),
        # a prompt, or a batch of prompts, of 4096 tokens
        _norm("norm_4096_tokens", "norm", 4096, 4096),
        # a training batch of 2 sequences of 1024
        _norm("norm_train_2048_tokens", "norm_train", 2048, 4096),
        # a small model's ragged batch, its stream in float32
        _norm("norm_train_ragged", "norm_train", 333, 1160, stream="f32"),
        # a decoding batch: one token each of 48 requests
        _cached("append_48_sequences", "append", 48, 1, 4096, 8, 4, 128),
        # two prompts, one of them the next part of a longer one
        _cached("append_prompts", "append", 2, 2048, 3001, 8, 4, 128),
        # one request with a long text behind it
        _cached("attend_1_sequence", "attend", 1, 1, 32768, 8, 4, 128),
        # a decoding batch of 48 requests, each as far as it is
        _cached("attend_48_sequences", "attend", 48, 1, 8192, 8, 4, 128),
        # a prompt of 4096 tokens
        _cached("attend_prompt", "attend", 1, 4096, 4096, 8, 4, 128),
        # parts of five prompts of a smaller model that looks 256 tokens back, short pages
        _cached("attend_parts_window", "attend", 5, 333, 2011, 3, 5, 64, page=16, window=256),
        # one request's logits, its text as its history
        _logits("logits_1_row", 1, 128256, 1000, 20, 0),
        # a decoding batch of 48 requests, half of them bound to one of 4 grammars
        _logits("logits_48_rows", 48, 128256, 4000, 100, 4),
    ]


def _log_int(rng, lo, hi, step=1):
    """step * lo .. step * hi in steps, spread over the logarithm."""
    return step * int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["norm", "norm_train", "append", "append", "attend", "attend", "attend", "logits"])
    if do in ("norm", "norm_train"):
        width = _log_int(rng, 8, 1024, 8)
        return _norm(None, do, _log_int(rng, 1, min(8192, 4096 * 4096 // width)), width, rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16", "none"]))
    if do == "logits":
        vocab = _log_int(rng, 1000, 128256)
        return _logits(None, _log_int(rng, 1, 64), vocab, _log_int(rng, 1, 8192), _log_int(rng, 1, 300), rng.choice([0, 0, 1, 4]))
    dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    heads, group = _log_int(rng, 1, 16), rng.choice([1, 2, 3, 4, 5, 8])
    if rng.random() < 0.6:      # a decoding batch
        sequences, new = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4])
        longest = _log_int(rng, 16, max(32, min(32768, (32 << 20) // (sequences * heads * dim))))
    else:                       # prompts, or parts of them
        sequences, new = _log_int(rng, 1, 6), _log_int(rng, 8, 2048)
        longest = max(new, _log_int(rng, 16, max(32, min(16384, (1 << 28) // (sequences * new * heads * group), (32 << 20) // (sequences * heads * dim)))))
    new = min(new, longest)
    return _cached(None, do, sequences, new, longest, heads, group, dim, page, rng.choice([0, 0, 0, 100, 256, 1024]), rng.choice(["f32", "f32", "bf16"]))


# ---------------------------------------------------------------------------- what a program has in hand
def _generator(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(9_000_000_011 + 1000 * (int(seed) % 1000003) + tag)
    return g


def _normal(shape, seed, tag, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=_generator(seed, tag), device=DEV, dtype=torch.float32) * std).to(dtype)


def _plan(case):
    """(new tokens, length with them) of every sequence."""
    plan = []
    for s in range(case["sequences"]):
        far = 1 - 0.75 * (s * 0.6180339887 % 1)
        new = max(1, int(case["new"] * (1 - 0.5 * (s * 0.7548776662 % 1))))
        plan.append((new, max(new, int(case["longest"] * far))))
    return plan


def _sequences(case, seed):
    """starts, lengths and the table of pages, in no order among the pool's; how many pages the pool has."""
    plan, page = _plan(case), case["page"]
    starts = [0]
    for new, _ in plan:
        starts.append(starts[-1] + new)
    need = [-(-length // page) for _, length in plan]
    pool, wide = sum(need) + 3, -(-case["longest"] // page)
    order = torch.randperm(pool, generator=_generator(seed, 100), device=DEV).to(torch.int32)
    table = torch.zeros((len(plan), wide), dtype=torch.int32, device=DEV)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return (torch.tensor(starts, dtype=torch.int32, device=DEV), torch.tensor([length for _, length in plan], dtype=torch.int32, device=DEV),
            table, pool)


def _scale_for(most):
    """The smallest power of two by which `most` fits the 448 of e4m3, at least 2^-100."""
    fraction, exponent = torch.frexp(most)
    exponent = torch.where(most > 0, exponent - 9 + (fraction > 0.875), -100).clamp(min=-100)
    return torch.ldexp(torch.ones_like(most), exponent)


def _pages(case, pool, seed, tag, values):
    """The pages' content from tokens before: e4m3 and a scale for each page and head.  Keys differ much from channel to channel."""
    shape = (pool, case["heads"], case["page"], case["dim"])
    x = _normal(shape, seed, tag)
    x *= torch.exp(_normal((1, case["heads"], 1, case["dim"]), seed, tag + 1, 0.5 if not values else 0.1))
    scale = _scale_for(x.abs().amax(dim=(2, 3)))
    x = (x / scale[:, :, None, None]).to(E4M3)
    return (x.view(torch.uint8).transpose(2, 3).contiguous().view(E4M3) if values else x), scale


def _inputs(case, seed):
    do = case["do"]
    st = {}
    if do in ("norm", "norm_train"):
        shape = (case["tokens"], case["width"])
        st["x"] = _normal(shape, seed, 0, 0.5, TYPES[case["x"]])
        st["weight"] = 1 + _normal((case["width"],), seed, 1, 0.2)
        st["residual"] = _normal(shape, seed, 2, 1.0, TYPES[case["stream"]]) if case["stream"] != "none" else None
        if do == "norm_train":
            st["grad_y"] = _normal(shape, seed, 3, 0.01, torch.bfloat16)
            # (what comes back along the stream)
            st["grad_total"] = _normal(shape, seed, 4, 0.01, torch.bfloat16) if st["residual"] is not None else None
        return st
    if do == "logits":
        rows, vocab = case["rows"], case["vocab"]
        st["logits"] = _normal((rows, vocab), seed, 10, 3.0)
        lens = [max(0, int(case["history"] * (1 - 0.9 * (r * 0.6180339887 % 1)))) for r in range(rows)]
        bias = [int(case["biases"] * (1 - (r * 0.7548776662 % 1))) for r in range(rows)]
        for name, of in (("history", lens), ("bias", bias)):
            starts = torch.tensor([0] + of, dtype=torch.int64).cumsum(0).to(torch.int32)
            st[name + "_starts"] = starts.to(DEV)
            # (texts have few words very often)
            u = torch.rand(int(starts[-1]), generator=_generator(seed, 11 + len(name)), device=DEV, dtype=torch.float64)
            rank = torch.exp(u * math.log(vocab)).long().clamp_(1, vocab) - 1
            st[name] = (rank * 2654435761 + int(seed) % 1000003) % vocab
        st["bias_values"] = _normal((st["bias"].numel(),), seed, 12, 2.0)
        g = _generator(seed, 13)
        st["repetition"] = 1 + torch.rand(rows, generator=g, device=DEV) * 0.3
        st["frequency"] = torch.rand(rows, generator=g, device=DEV) * 0.5
        st["presence"] = torch.rand(rows, generator=g, device=DEV) * 0.5
        if case["masks"]:
            words = -(-vocab // 32)
            st["masks"] = torch.randint(-2 ** 31, 2 ** 31, (case["masks"], words), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
            st["mask_ids"] = torch.randint(-case["masks"], case["masks"], (rows,), generator=g, device=DEV).clamp_(min=-1).to(torch.int32)
        else:
            st["masks"] = st["mask_ids"] = None
        return st
    st["starts"], st["lengths"], st["table"], pool = _sequences(case, seed)
    st["k_pages"], st["k_scales"] = _pages(case, pool, seed, 20, False)
    st["v_pages"], st["v_scales"] = _pages(case, pool, seed, 22, True)
    tokens, heads, dim = sum(new for new, _ in _plan(case)), case["heads"], case["dim"]
    if do == "attend":
        st["q"] = _normal((tokens, heads * case["group"], dim), seed, 24, 1.0, torch.bfloat16)
        return st
    # one projection's result: queries, keys and values side by side
    rows = _normal((tokens, heads * (case["group"] + 2), dim), seed, 25, 1.0, TYPES[case["x"]])
    st["q"], st["k"], st["v"] = rows.split([heads * case["group"], heads, heads], dim=1)
    at = torch.arange(st["table"].shape[1] * case["page"], dtype=torch.float64, device=DEV)
    angle = at[:, None] * 500000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEV) / dim)
    st["rotary"] = torch.cat([angle.cos(), angle.sin()], dim=1).float()
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if own and "table" in st:
        from paper_2410_20650_amd import binding as nz
        st["cache"] = nz.KeyValueCache(st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"])
        st["sequences"] = nz.Sequences(st["starts"], st["lengths"], st["table"])
    return st


# ---------------------------------------------------------------------------- one pass
def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    from paper_2410_20650_amd import binding as nz
    case = st["case"]
    do = case["do"]
    if do in ("norm", "norm_train"):
        out = nz.neuzip_norm(st["x"], st["weight"], EPS, st["residual"])
        y, total = out if st["residual"] is not None else (out, st["x"])
        if do == "norm":
            return [y, total]
        return [y, total, *nz.neuzip_norm_backward(total, st["weight"], st["grad_y"], EPS, st["grad_total"])]
    if do == "append":
        q = nz.neuzip_cache_append(st["cache"], st["sequences"], st["k"], st["v"], st["q"], st["rotary"])
        return {"q": q, "k": st["k_pages"], "v": st["v_pages"], "k_scales": st["k_scales"], "v_scales": st["v_scales"]}
    if do == "attend":
        return nz.neuzip_cache_attention(st["cache"], st["sequences"], st["q"], window=case["window"])
    return nz.neuzip_logits(st["logits"], st["history"], st["history_starts"], st["repetition"], st["frequency"], st["presence"], st["bias"],
                            st["bias_values"], st["bias_starts"], st["masks"], st["mask_ids"])


def _plain(st):
    case = st["case"]
    do = case["do"]
    if do in ("norm", "norm_train"):
        return _plain_norm(st, do == "norm_train")
    return {"append": _plain_append, "attend": _plain_attend, "logits": _plain_logits}[do](st)


def _plain_norm(st, train):
    w = st["weight"]
    total = st["x"]
    if st["residual"] is not None:
        total = (st["x"].float() + st["residual"].float()).to(st["residual"].dtype)
    s = total.float()
    inv = 1.0 / torch.sqrt((s * s).mean(dim=1, keepdim=True) + EPS)
    unit = s * inv
    y = (unit * w).to(torch.bfloat16)
    if not train:
        return [y, total]
    gy = st["grad_y"].float()
    g = gy * w
    gs = inv * (g - unit * (g * unit).mean(dim=1, keepdim=True))
    if st["grad_total"] is not None:
        gs = gs + st["grad_total"].float()
    return [y, total, gs.to(torch.bfloat16), (gy * unit).sum(dim=0)]


def _tokens_of(st):
    """Each token's sequence and position."""
    t = torch.arange(st["q"].shape[0], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(st["starts"][1:], t, right=True)
    start, end = st["starts"][:-1], st["starts"][1:]
    return seq, (st["lengths"] - (end - start))[seq].long() + (t - start[seq]).long()


def _rotated(x, at):
    half = x.shape[-1] // 2
    cos, sin = at[:, None, :half], at[:, None, half:]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_append(st):
    case = st["case"]
    page = case["page"]
    seq, pos = _tokens_of(st)
    at = st["rotary"][pos]
    q = _rotated(st["q"].float(), at).to(torch.bfloat16)
    to, slot = st["table"][seq, pos // page].long(), pos % page
    first = (st["lengths"] - (st["starts"][1:] - st["starts"][:-1])).long()     # of the new tokens' positions
    begun = st["table"][torch.arange(first.numel(), device=DEV), first // page].long()
    stay = first % page                                                         # tokens of that page that were there before
    for name, x, turn in (("k", _rotated(st["k"].float(), at), False), ("v", st["v"].float(), True)):
        held, scales = st[name + "_pages"].view(torch.uint8), st[name + "_scales"]
        most = torch.zeros_like(scales).scatter_reduce_(0, to[:, None].expand(-1, case["heads"]), x.abs().amax(dim=-1), "amax")
        touched = torch.zeros(scales.shape[0], dtype=torch.bool, device=DEV)
        touched[to] = True
        old = torch.zeros_like(scales)
        old[begun] = torch.where((stay > 0)[:, None], scales[begun], old[begun])
        new = torch.where(touched[:, None], torch.maximum(_scale_for(most), old), scales)
        kept = held[begun].view(E4M3).float() * (scales[begun] / new[begun])[:, :, None, None]
        here = torch.arange(page, device=DEV) < stay[:, None]
        here = here[:, None, None, :] if turn else here[:, None, :, None]
        held[begun] = torch.where(here, kept.to(E4M3).view(torch.uint8), held[begun])
        coded = (x / new[to][:, :, None]).to(E4M3).view(torch.uint8)
        if turn:
            held[to, :, :, slot] = coded
        else:
            held[to, :, slot] = coded
        scales.copy_(new)
    return {"q": q, "k": st["k_pages"], "v": st["v_pages"], "k_scales": st["k_scales"], "v_scales": st["v_scales"]}


def _plain_attend(st):
    case = st["case"]
    page, dim, heads, group = case["page"], case["dim"], case["heads"], case["group"]
    starts, lengths, table = st["starts"].long(), st["lengths"].long(), st["table"].long()
    n, wide = table.shape
    k = (st["k_pages"].float() * st["k_scales"][:, :, None, None])[table]            # sequence, page, head, token, feature
    v = (st["v_pages"].float() * st["v_scales"][:, :, None, None])[table]            # ... feature, token
    k = k.permute(0, 2, 4, 1, 3).reshape(n * heads, dim, wide * page)
    v = v.permute(0, 2, 1, 4, 3).reshape(n * heads, wide * page, dim)
    counts = starts[1:] - starts[:-1]
    seq, pos = _tokens_of(st)
    row = torch.arange(pos.numel(), device=DEV) - starts[:-1][seq]
    most = case["new"]
    q = torch.zeros((n, most, heads, group, dim), device=DEV)
    q[seq, row] = st["q"].float().view(-1, heads, group, dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(n * heads, most * group, dim)
    score = torch.bmm(q, k).view(n, heads, most, group, wide * page) / math.sqrt(dim)
    key = torch.arange(wide * page, device=DEV)
    at = (lengths - counts)[:, None] + torch.arange(most, device=DEV)
    seen = (key <= at[:, :, None]) & (key < lengths[:, None, None])
    if case["window"]:
        seen &= key > at[:, :, None] - case["window"]
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    out = torch.bmm(p.view(n * heads, most * group, wide * page), v).view(n, heads, most, group, dim)
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out.permute(0, 2, 1, 3, 4)[seq, row].reshape(-1, heads * group, dim).to(torch.bfloat16)


def _rows_of(starts, count):
    return torch.searchsorted(starts[1:], torch.arange(count, device=DEV, dtype=torch.int32), right=True)


def _plain_logits(st):
    x = st["logits"]
    rows, vocab = x.shape
    count = torch.zeros((rows, vocab), dtype=torch.int32, device=DEV)
    count.view(-1).index_add_(0, _rows_of(st["history_starts"], st["history"].numel()) * vocab + st["history"],
                              torch.ones(st["history"].numel(), dtype=torch.int32, device=DEV))
    there = count > 0
    rep = st["repetition"][:, None]
    x = torch.where(there, torch.where(x > 0, x / rep, x * rep), x)
    x = x - st["frequency"][:, None] * count
    x = torch.where(there, x - st["presence"][:, None], x)
    # a token that is named twice: the later entry counts
    entries = torch.arange(st["bias"].numel(), device=DEV)
    last = torch.full((rows * vocab,), -1, dtype=torch.int64, device=DEV)
    last.scatter_reduce_(0, _rows_of(st["bias_starts"], entries.numel()) * vocab + st["bias"], entries, "amax")
    last = last.view(rows, vocab)
    values = torch.cat([st["bias_values"], torch.zeros(1, device=DEV)])     # (-1: the zero behind them)
    x = x + values[last]
    if st["masks"] is not None:
        at = torch.arange(vocab, device=DEV)
        ids = st["mask_ids"].long()
        allowed = (st["masks"][ids.clamp(min=0)][:, at >> 5] >> (at & 31).to(torch.int32)) & 1
        x = torch.where((allowed == 0) & (ids >= 0)[:, None], torch.full_like(x, -math.inf), x)
    return x


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    do = case["do"]
    if do in ("norm", "norm_train"):
        n, w = case["tokens"] * case["width"], case["width"]
        size = {"f32": 4, "bf16": 2, "none": 0}
        held = size[case["stream"]] or size[case["x"]]
        forward = n * (size[case["x"]] + 2 * size[case["stream"]] + 2) + 4 * w
        if do == "norm":
            return {"bytes": forward, "flops": 5 * n}
        return {"bytes": forward + n * (held + 2 + 2 + (2 if case["stream"] != "none" else 0)) + 8 * w, "flops": 16 * n}
    if do == "logits":
        n = case["rows"] * case["vocab"]
        # (the histories are about half of the longest, the biases too)
        return {"bytes": 8 * n + case["masks"] * case["vocab"] // 8 + case["rows"] * (8 * case["history"] + 12 * case["biases"]) // 2, "flops": 6 * n}
    plan, heads, dim, group = _plan(case), case["heads"], case["dim"], case["group"]
    tokens = sum(new for new, _ in plan)
    if do == "append":
        size = {"f32": 4, "bf16": 2}[case["x"]]
        return {"bytes": tokens * heads * dim * ((group + 2) * size + 2 * group + 2) + 4 * tokens * dim, "flops": 4 * tokens * heads * dim * (group + 2)}
    window = case["window"] or 1 << 40
    read = sum(min(length, new + window - 1) for new, length in plan)
    # (position p sees min(p + 1, window) keys)
    pairs = sum(sum(min(p + 1, window) for p in range(length - new, length)) for new, length in plan)
    return {"bytes": 2 * read * heads * dim + 4 * tokens * heads * group * dim, "flops": 4 * dim * heads * group * pairs}


# ---------------------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    do = case["do"]
    st = _inputs(case, seed)
    if do in ("norm", "norm_train"):
        total = st["x"]
        if st["residual"] is not None:      # the stream as it is held, which is what the norm sees
            total = (st["x"].double() + st["residual"].double()).to(st["residual"].dtype)
        s, w = total.double(), st["weight"].double()
        power = s.square().sum(dim=1, keepdim=True) / case["width"] + EPS
        y = s * power.rsqrt() * w
        if do == "norm":
            return [y, total.double()]
        gy = st["grad_y"].double()
        # d/ds of sum(gy * w * s * power^-1/2)
        gs = gy * w * power.rsqrt() - s * (gy * w * s).sum(dim=1, keepdim=True) * power ** -1.5 / case["width"]
        if st["grad_total"] is not None:
            gs += st["grad_total"].double()
        return [y, total.double(), gs, torch.einsum("tw,tw->w", gy, s * power.rsqrt())]
    return {"append": _exact_append, "attend": _exact_attend, "logits": _exact_logits}[do](case, st)


def _exact_e4m3(x):
    """The nearest value of 3 bits behind the leading one, down to 2^-6, and of steps of 2^-9 below; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(case, st):
    page, dim, plan = case["page"], case["dim"], _plan(case)
    pages = {"k": st["k_pages"].double(), "v": st["v_pages"].double().transpose(2, 3).contiguous()}
    scales = {"k": st["k_scales"].double(), "v": st["v_scales"].double()}
    rotary = st["rotary"].double()
    table = st["table"].tolist()
    turned = []
    at = 0
    for s, (new, length) in enumerate(plan):
        first = length - new
        c, d = (t[:, None] for t in rotary[first:length].split(dim // 2, dim=1))
        z = {}
        for name in ("q", "k"):
            x = st[name][at:at + new].double()
            a, b = x[..., :dim // 2], x[..., dim // 2:]
            z[name] = torch.cat([a * c - b * d, a * d + b * c], dim=-1)
        z["v"] = st["v"][at:at + new].double()
        turned.append(z["q"])
        for number in range(first // page, (length - 1) // page + 1):
            to, begin = table[s][number], max(first, number * page)
            end = min(length, (number + 1) * page)
            for name in ("k", "v"):
                x = z[name][begin - first:end - first].transpose(0, 1)      # head, token, feature
                most = x.abs().amax(dim=(1, 2))
                # the least power of two with most <= 448 of it
                fit = torch.exp2(torch.ceil(torch.log2(most / 448)).clamp(min=-100.0))
                inside = begin - number * page
                if inside > 0:
                    fit = torch.maximum(fit, scales[name][to])
                    pages[name][to, :, :inside] = _exact_e4m3(pages[name][to, :, :inside] * (scales[name][to] / fit)[:, None, None])
                scales[name][to] = fit
                pages[name][to, :, inside:inside + end - begin] = _exact_e4m3(x / fit[:, None, None])
        at += new
    return {"q": torch.cat(turned), "k": pages["k"], "v": pages["v"].transpose(2, 3).contiguous(), "k_scales": scales["k"], "v_scales": scales["v"]}


def _exact_attend(case, st):
    page, dim, heads, group, window = case["page"], case["dim"], case["heads"], case["group"], case["window"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for s, (new, length) in enumerate(_plan(case)):
        to = st["table"][s, :-(-length // page)].long()
        query = torch.arange(length - new, length, device=DEV)[:, None]
        key = torch.arange(length, device=DEV)
        hidden = key > query
        if window:
            hidden = hidden | (key + window <= query)
        for h in range(heads):
            k = (st["k_pages"].view(torch.uint8)[to, h].view(E4M3).double() * st["k_scales"][to, h].double()[:, None, None]).reshape(-1, dim)[:length]
            v = st["v_pages"].view(torch.uint8)[to, h].view(E4M3).double() * st["v_scales"][to, h].double()[:, None, None]
            v = v.transpose(1, 2).reshape(-1, dim)[:length]
            for j in range(h * group, (h + 1) * group):
                weight = torch.matmul(st["q"][at:at + new, j].double(), k.t()) * dim ** -0.5
                weight = torch.softmax(weight.masked_fill_(hidden, -math.inf), dim=1)
                out[at:at + new, j] = torch.matmul(weight, v)
        at += new
    return out


def _exact_logits(case, st):
    vocab = case["vocab"]
    out = st["logits"].double()
    history, bias = st["history_starts"].tolist(), st["bias_starts"].tolist()
    shift = torch.arange(32, device=DEV)
    for r in range(case["rows"]):
        x = out[r]
        count = torch.bincount(st["history"][history[r]:history[r + 1]], minlength=vocab).double()
        had = count > 0
        rep = float(st["repetition"][r])
        x[had] *= torch.where(x[had] > 0, 1.0 / rep, rep)
        x -= count * float(st["frequency"][r]) + had * float(st["presence"][r])
        named = dict(zip(st["bias"][bias[r]:bias[r + 1]].tolist(), st["bias_values"][bias[r]:bias[r + 1]].tolist()))
        if named:
            x[torch.tensor(list(named), device=DEV)] += torch.tensor(list(named.values()), dtype=torch.float64, device=DEV)
        if case["masks"] and int(st["mask_ids"][r]) >= 0:
            bits = (st["masks"][int(st["mask_ids"][r])].long()[:, None] >> shift) & 1
            x[bits.reshape(-1)[:vocab] == 0] = -math.inf
    return out
