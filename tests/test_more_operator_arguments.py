"""What the calls of the norm, the cache, its attention and the logits refuse without a GPU: the binding by the tensors it is given (stand-ins, and nothing
reaches the library), the library by its arguments, before any device work; and whose memory the calls' own tensors are of.
"""
import ctypes
import math

import pytest
import torch

from paper_2410_20650_amd import binding as nz
from test_operator_memory import CURRENT, STREAMS, expected, made  # noqa: F401 (a fixture)

BF, F32, I32, I64, E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.int64, torch.float8_e4m3fn
TOKENS, WIDTH, HEADS, GROUP, DIM, PAGE, PAGES, SEQUENCES, WIDE, VOCAB = 6, 256, 2, 3, 64, 16, 9, 4, 5, 100


class Stub:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype=BF, device=0, stride=None):
        self.shape, self.dtype, self.is_cuda, self.device = torch.Size(shape), dtype, device >= 0, torch.device("cuda", max(device, 0))
        self._device = device
        whole = [math.prod(shape[i + 1:]) for i in range(len(shape))]
        self._stride = tuple(stride or whole)
        self._contiguous = all(s == 1 or a == b for s, a, b in zip(shape, self._stride, whole))

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def get_device(self):
        return self._device

    def stride(self):
        return self._stride

    def is_contiguous(self):
        return self._contiguous

    def element_size(self):
        return self.dtype.itemsize

    def data_ptr(self):
        return 0x1000


@pytest.fixture
def called(monkeypatch):
    """The names of the library's functions that are called."""
    names = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: names.append(name) or 0

    monkeypatch.setattr(nz, "_lib", Library())
    monkeypatch.setattr(nz, "_stream_handle", lambda stream, device=None: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return names


def reached(names):
    return [n for n in names if not n.endswith("_scratch_bytes")]


def cache(k=Stub((PAGES, HEADS, PAGE, DIM), E4M3), v=Stub((PAGES, HEADS, DIM, PAGE), E4M3), k_scales=Stub((PAGES, HEADS), F32), v_scales=Stub((PAGES, HEADS), F32)):
    return nz.KeyValueCache(k, v, k_scales, v_scales)


def sequences(starts=Stub((SEQUENCES + 1,), I32), lengths=Stub((SEQUENCES,), I32), table=Stub((SEQUENCES, WIDE), I32)):
    return nz.Sequences(starts, lengths, table)


def norm(x=Stub((TOKENS, WIDTH), F32), weight=Stub((WIDTH,), F32), residual=Stub((TOKENS, WIDTH)), y=Stub((TOKENS, WIDTH)), total=Stub((TOKENS, WIDTH))):
    nz.neuzip_norm(x, weight, 1e-5, residual, y, total)


def norm_backward(total=Stub((TOKENS, WIDTH)), weight=Stub((WIDTH,), F32), grad_y=Stub((TOKENS, WIDTH)), grad_total=Stub((TOKENS, WIDTH)),
                  grad_x=Stub((TOKENS, WIDTH)), grad_weight=Stub((WIDTH,), F32), scratch=Stub((4096,), torch.uint8)):
    nz.neuzip_norm_backward(total, weight, grad_y, 1e-5, grad_total, grad_x, grad_weight, scratch)


def cache_append(k=Stub((TOKENS, HEADS, DIM), F32), v=Stub((TOKENS, HEADS, DIM), F32), q=Stub((TOKENS, HEADS * GROUP, DIM), F32),
                 rotary=Stub((WIDE * PAGE, DIM), F32), q_out=Stub((TOKENS, HEADS * GROUP, DIM))):
    nz.neuzip_cache_append(cache(), sequences(), k, v, q, rotary, q_out)


def cache_attention(q=Stub((TOKENS, HEADS * GROUP, DIM)), out=Stub((TOKENS, HEADS * GROUP, DIM)), scratch=Stub((4096,), torch.uint8)):
    nz.neuzip_cache_attention(cache(), sequences(), q, out=out, scratch=scratch)


ROWS = Stub((TOKENS,), F32)


def logits(logits=Stub((TOKENS, VOCAB), F32), history=Stub((50,), I64), history_starts=Stub((TOKENS + 1,), I32), repetition=ROWS, frequency=ROWS, presence=ROWS,
           bias=Stub((7,), I64), bias_values=Stub((7,), F32), bias_starts=Stub((TOKENS + 1,), I32), masks=Stub((2, 4), I32), mask_ids=Stub((TOKENS,), I32),
           out=Stub((TOKENS, VOCAB), F32)):
    nz.neuzip_logits(logits, history, history_starts, repetition, frequency, presence, bias, bias_values, bias_starts, masks, mask_ids, out)


CALLS = {
    cache: dict(k=((PAGES, HEADS, PAGE, DIM), E4M3), v=((PAGES, HEADS, DIM, PAGE), E4M3), k_scales=((PAGES, HEADS), F32), v_scales=((PAGES, HEADS), F32)),
    sequences: dict(starts=((SEQUENCES + 1,), I32), lengths=((SEQUENCES,), I32), table=((SEQUENCES, WIDE), I32)),
    norm: dict(x=((TOKENS, WIDTH), F32), weight=((WIDTH,), F32), residual=((TOKENS, WIDTH), BF), y=((TOKENS, WIDTH), BF), total=((TOKENS, WIDTH), BF)),
    norm_backward: dict(total=((TOKENS, WIDTH), BF), weight=((WIDTH,), F32), grad_y=((TOKENS, WIDTH), BF), grad_total=((TOKENS, WIDTH), BF),
                        grad_x=((TOKENS, WIDTH), BF), grad_weight=((WIDTH,), F32)),
    cache_append: dict(k=((TOKENS, HEADS, DIM), F32), v=((TOKENS, HEADS, DIM), F32), q=((TOKENS, HEADS * GROUP, DIM), F32), rotary=((WIDE * PAGE, DIM), F32),
                       q_out=((TOKENS, HEADS * GROUP, DIM), BF)),
    cache_attention: dict(q=((TOKENS, HEADS * GROUP, DIM), BF), out=((TOKENS, HEADS * GROUP, DIM), BF)),
    logits: dict(logits=((TOKENS, VOCAB), F32), history=((50,), I64), history_starts=((TOKENS + 1,), I32), repetition=((TOKENS,), F32), frequency=((TOKENS,), F32),
                 presence=((TOKENS,), F32), bias=((7,), I64), bias_values=((7,), F32), bias_starts=((TOKENS + 1,), I32), masks=((2, 4), I32),
                 mask_ids=((TOKENS,), I32), out=((TOKENS, VOCAB), F32)),
}


@pytest.mark.parametrize("call", CALLS)
def test_accepted(called, call):
    call()
    assert reached(called) == ([] if call in (cache, sequences) else ["neuzip_" + call.__name__])


@pytest.mark.parametrize("call, name", [(c, n) for c, names in CALLS.items() for n in names])
def test_refused(called, call, name):
    shape, dtype = CALLS[call][name]
    bad = [(TypeError, Stub(shape, torch.float64)), (TypeError, Stub(shape, dtype, device=-1)), (ValueError, Stub((*shape[:-1], shape[-1] + 1), dtype)),
           (ValueError, Stub(shape, dtype, device=1))]
    if len(shape) > 1:
        gaps = [2 * math.prod(shape[i + 1:]) for i in range(len(shape))]
        bad.append(((TypeError, ValueError), Stub(shape, dtype, stride=gaps)))      # the elements lie apart
    for error, stub in bad:
        if (call, name) in ((sequences, "table"), (logits, "history")) and error is ValueError and stub.get_device() == 0:
            continue    # (any table will do, and any number of tokens)
        with pytest.raises(error):
            call(**{name: stub})
    assert reached(called) == []


@pytest.mark.parametrize("bad", [dict(window=-1), dict(window=1 << 32), dict(longest=-1), dict(longest=1 << 64)])
def test_numbers_of_tokens_that_are_none(called, bad):
    with pytest.raises(ValueError):
        nz.neuzip_cache_attention(cache(), sequences(), Stub((TOKENS, HEADS * GROUP, DIM)), **bad)
    assert reached(called) == []


def test_rows_that_lie_apart(called):
    """Parts of a projection's rows are taken as they are, if rows begin on 16 bytes; a row's own elements have no gaps."""
    part = (TOKENS, HEADS * DIM)
    for stride, dtype, fine in (((WIDTH * 3, 1), F32, True), ((WIDTH * 3 + 2, 1), F32, False), ((HEADS * DIM - 4, 1), F32, False), ((WIDTH * 3, 2), F32, False),
                                ((WIDTH * 3 + 4, 1), BF, False), ((WIDTH * 3 + 8, 1), BF, True)):
        k, v = Stub(part, dtype, stride=stride), Stub(part, dtype)
        if fine:
            nz.neuzip_cache_append(cache(), sequences(), k, v)
        else:
            with pytest.raises(ValueError):
                nz.neuzip_cache_append(cache(), sequences(), k, v)
    nz.neuzip_cache_attention(cache(), sequences(), Stub((TOKENS, HEADS * GROUP, DIM), stride=(5000, DIM, 1)), out=Stub((TOKENS, HEADS * GROUP, DIM)))
    assert reached(called) == ["neuzip_cache_append"] * 2 + ["neuzip_cache_attention"]


def test_what_belongs_together(called):
    refused = [lambda: norm(residual=None), lambda: cache_append(q=None), lambda: cache_append(v=Stub((TOKENS + 1, HEADS, DIM), F32)),
               lambda: cache_append(q=Stub((TOKENS - 1, HEADS, DIM), F32)), lambda: cache_append(rotary=Stub((WIDE * PAGE - 1, DIM), F32)),
               lambda: cache_attention(q=Stub((TOKENS, HEADS * GROUP + 1, DIM))), lambda: logits(history=None), lambda: logits(history_starts=None),
               lambda: logits(bias=None), lambda: logits(bias_values=None), lambda: logits(masks=None), lambda: logits(mask_ids=None),
               lambda: cache(k=Stub((PAGES, HEADS, 20, DIM), E4M3)), lambda: cache(k=Stub((PAGES, HEADS, PAGE, 96), E4M3)),
               lambda: cache(v=Stub((PAGES, HEADS, PAGE, DIM), E4M3))]
    for call in refused:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        cache_append(v=Stub((TOKENS, HEADS, DIM), BF))      # one type for all three
    assert reached(called) == []


def test_scratch_memory_and_devices(called, monkeypatch):
    for call in (norm_backward, cache_attention):
        for stub in (Stub((64,), torch.uint8, device=-1), Stub((64, 2), torch.uint8, stride=(4, 1))):
            with pytest.raises(TypeError):
                call(scratch=stub)
        with pytest.raises(ValueError):
            call(scratch=Stub((64,), torch.uint8, device=1))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (norm, norm_backward, cache_append, cache_attention, logits):
        with pytest.raises(ValueError):
            call()
    assert reached(called) == []


# results that the caller has not brought along, and how many tensors with the scratch memory
OF_ITS_OWN = {
    "norm": (1, lambda s: nz.neuzip_norm(Stub((TOKENS, WIDTH), F32), Stub((WIDTH,), F32), 1e-5, stream=s)),
    "norm, stream": (2, lambda s: nz.neuzip_norm(Stub((TOKENS, WIDTH), F32), Stub((WIDTH,), F32), 1e-5, Stub((TOKENS, WIDTH)), stream=s)),
    "norm_backward": (3, lambda s: nz.neuzip_norm_backward(Stub((TOKENS, WIDTH)), Stub((WIDTH,), F32), Stub((TOKENS, WIDTH)), 1e-5, stream=s)),
    "cache_append": (1, lambda s: nz.neuzip_cache_append(cache(), sequences(), *(Stub((TOKENS, HEADS, DIM)) for _ in range(3)), stream=s)),
    "cache_attention": (2, lambda s: nz.neuzip_cache_attention(cache(), sequences(), Stub((TOKENS, HEADS, DIM)), stream=s)),
    "logits": (1, lambda s: nz.neuzip_logits(Stub((TOKENS, VOCAB), F32), stream=s)),
}


@pytest.mark.parametrize("stream", STREAMS)
@pytest.mark.parametrize("name", OF_ITS_OWN)
def test_whose_memory(made, monkeypatch, name, stream):     # noqa: F811
    make = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *shape, **kw: make(*shape, **kw) and Stub(shape[0] if isinstance(shape[0], tuple) else shape, kw["dtype"]))
    monkeypatch.setattr(torch, "empty_like", lambda t, dtype: torch.empty(tuple(t.shape), dtype=dtype, device=t.device))
    count, call = OF_ITS_OWN[name]
    call(stream)
    assert made == [expected(stream)] * count and CURRENT != 0x22


# ---------------------------------------------------------------------------- the library itself
SOME, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)


def c_cache(**other):
    return nz._Cache(**{**dict(d_k=0x1000, d_v=0x1000, d_k_scales=0x1000, d_v_scales=0x1000, pages=9, heads=2, head_dim=64, page_tokens=16), **other})


def c_sequences(**other):
    return nz._Sequences(**{**dict(d_starts=0x1000, d_lengths=0x1000, d_table=0x1000, count=4, table_width=5), **other})


def append(c=None, s=None, type_=nz.F32, k=SOME, k_row=128, v=SOME, v_row=128, q=None, q_row=0, q_heads=0, q_out=None, rotary=None, rotary_rows=0, rows=0):
    return nz.library().neuzip_cache_append(c or c_cache(), s or c_sequences(), type_, k, k_row, v, v_row, q, q_row, q_heads, q_out, rotary, rotary_rows, rows, None)


def attention(c=None, s=None, q=SOME, q_row=384, q_heads=6, rows=3, scale=0.125, window=0, longest=0, out=SOME, scratch=None, room=0):
    return nz.library().neuzip_cache_attention(c or c_cache(), s or c_sequences(), q, q_row, q_heads, rows, scale, window, longest, out, scratch, room, None)


BAD_CACHES = [dict(d_k=0), dict(d_v=0), dict(d_k_scales=0), dict(d_v_scales=0), dict(d_k=0x1008), dict(d_v=0x1004), dict(d_k_scales=0x1002), dict(pages=0),
              dict(pages=1 << 31), dict(heads=0), dict(head_dim=96), dict(head_dim=0), dict(page_tokens=0), dict(page_tokens=24), dict(page_tokens=256)]
BAD_SEQUENCES = [dict(d_starts=0), dict(d_lengths=0), dict(d_table=0), dict(d_table=0x1002), dict(table_width=0), dict(count=1 << 24), dict(table_width=1 << 27)]


def test_the_library_refuses_caches_and_sequences():
    for other in BAD_CACHES:
        assert append(c_cache(**other), rows=3) == nz.EINVAL and attention(c_cache(**other)) == nz.EINVAL, other
        assert nz.library().neuzip_cache_attention_scratch_bytes(c_cache(**other), c_sequences(), 6, 3, 0, 0) == 0
    for other in BAD_SEQUENCES:
        assert append(s=c_sequences(**other), rows=3) == nz.EINVAL and attention(s=c_sequences(**other)) == nz.EINVAL, other
    lib = nz.library()
    assert lib.neuzip_cache_append(None, c_sequences(), 1, SOME, 128, SOME, 128, None, 0, 0, None, None, 0, 3, None) == nz.EINVAL
    assert lib.neuzip_cache_attention(c_cache(), None, SOME, 384, 6, 3, 0.125, 0, 0, SOME, None, 0, None) == nz.EINVAL


def test_the_library_refuses_appends():
    assert append() == append(s=c_sequences(count=0, d_starts=0, d_lengths=0, d_table=0), rows=3) == nz.OK      # nothing to do
    for other in (dict(type_=nz.F16), dict(type_=7), dict(k=None), dict(v=None), dict(k=ODD), dict(k_row=124), dict(v_row=130), dict(q=SOME), dict(q_out=SOME),
                  dict(q=SOME, q_out=SOME, q_heads=0, q_row=384), dict(q=SOME, q_out=SOME, q_heads=6, q_row=380), dict(q=SOME, q_out=ODD, q_heads=6, q_row=384),
                  dict(rotary=SOME, rotary_rows=79), dict(rotary=ODD, rotary_rows=80), dict(rows=1 << 31), dict(type_=nz.BF16, k_row=132)):
        assert append(**{"rows": 3, **other}) == nz.EINVAL, other
    assert append(c_cache(heads=1 << 16), k_row=1 << 22, v_row=1 << 22, rows=3) == nz.EUNSUPPORTED
    assert append(rows=(1 << 31) - 1) == nz.EUNSUPPORTED


def test_the_library_refuses_attention():
    assert attention(rows=0) == nz.OK
    for other in (dict(q=None), dict(out=None), dict(q=ODD), dict(out=ODD), dict(q_heads=0), dict(q_heads=5), dict(q_row=383), dict(q_row=376), dict(scale=0.0),
                  dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(scratch=ODD)):
        assert attention(**other) == nz.EINVAL, other
    assert attention(rows=1 << 25) == nz.EUNSUPPORTED
    s = c_sequences(count=1, table_width=1000)
    room = nz.library().neuzip_cache_attention_scratch_bytes(c_cache(), s, 6, 3, 0, 0)
    assert room > 0 and attention(s=s) == attention(s=s, scratch=SOME, room=room - 1) == nz.EINVAL
    # a window, or an upper bound of the lengths, leaves nothing to split
    for window, longest in ((100, 0), (0, 500)):
        assert nz.library().neuzip_cache_attention_scratch_bytes(c_cache(), s, 6, 3, window, longest) == 0


def test_the_library_refuses_norms():
    forward, backward = nz.library().neuzip_norm, nz.library().neuzip_norm_backward

    def norm_of(x=SOME, x_type=1, residual=SOME, total=SOME, total_type=0, weight=SOME, tokens=3, width=256, eps=1e-5, y=SOME):
        return forward(x, x_type, residual, total, total_type, weight, tokens, width, eps, y, None)

    def back_of(total=SOME, total_type=0, weight=SOME, grad_y=SOME, grad_total=None, tokens=3, width=256, eps=1e-5, grad_x=SOME, grad_weight=None, scratch=None, room=0):
        return backward(total, total_type, weight, grad_y, grad_total, tokens, width, eps, grad_x, grad_weight, scratch, room, None)

    assert norm_of(tokens=0) == nz.OK and back_of(tokens=0) == nz.OK and back_of(grad_x=None) == nz.OK
    for other in (dict(x=None), dict(weight=None), dict(y=None), dict(x=ODD), dict(total=ODD), dict(residual=None), dict(total=None), dict(x_type=2), dict(total_type=2),
                  dict(residual=None, total=None), dict(width=0), dict(width=12), dict(width=16392), dict(eps=-1.0), dict(eps=math.nan)):
        assert norm_of(**other) == nz.EINVAL, other
    for other in (dict(total=None), dict(weight=None), dict(grad_y=None), dict(grad_y=ODD), dict(grad_total=ODD), dict(grad_x=ODD), dict(total_type=2), dict(width=4),
                  dict(width=16392), dict(eps=math.nan), dict(tokens=0, grad_weight=SOME, weight=None)):
        assert back_of(**other) == nz.EINVAL, other
    room = nz.neuzip_norm_backward_scratch_bytes(300, 256)
    assert room > 0 and nz.neuzip_norm_backward_scratch_bytes(3, 256) == 0      # (one workgroup's part is the whole)
    for scratch, size in ((None, 0), (SOME, room - 1), (ODD, room)):
        assert back_of(tokens=300, grad_weight=SOME, scratch=scratch, room=size) == nz.EINVAL
    assert norm_of(tokens=1 << 24) == back_of(tokens=1 << 24) == nz.EUNSUPPORTED


def test_the_library_refuses_logits():
    call = nz.library().neuzip_logits

    def logits_of(x=SOME, rows=2, vocab=100, history=None, tokens=0, starts=None, repetition=None, bias=None, values=None, entries=0, bias_starts=None, masks=None,
                  count=0, ids=None, out=SOME):
        return call(x, rows, vocab, history, tokens, starts, repetition, None, None, bias, values, entries, bias_starts, masks, count, ids, out, None)

    assert logits_of(rows=0) == nz.OK
    off = ctypes.c_void_p(0x1002)
    for other in (dict(x=None), dict(out=None), dict(x=off), dict(out=off), dict(vocab=0), dict(tokens=5), dict(tokens=5, history=SOME), dict(tokens=5, starts=SOME),
                  dict(history=ctypes.c_void_p(0x1004), tokens=5, starts=SOME), dict(repetition=off), dict(entries=3), dict(entries=3, bias=SOME, values=SOME),
                  dict(masks=SOME, count=1), dict(ids=SOME), dict(masks=SOME, ids=SOME), dict(masks=SOME, ids=SOME, count=1 << 31)):
        assert logits_of(**other) == nz.EINVAL, other
    assert logits_of(rows=65536) == logits_of(vocab=1 << 31) == nz.EUNSUPPORTED
