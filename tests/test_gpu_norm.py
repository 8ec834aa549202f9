"""The root-mean-square norm with the residual's addition against 64 bits (-m gpu), forward and backward.

Bounds.  The sum x + residual is one binary32 addition rounded to the stream's type: compared bit for bit.  A row's sum of squares has at most
width / 512 + 20 additions one behind the other, each half a step (2^-24); n is off by half of that and a few roundings, so y by at most
(width / 1024 + 20) 2^-24 relative before it is rounded to bf16 (2^-8).  The backward pass' second sum, of g * total, is off by as much of the sum of its
terms' sizes.  A column's sum over the tokens is off by at most (tokens + 20) 2^-24 of the sum of its terms' sizes.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ULP = 2.0 ** -24


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def normal(*shape, seed, std=1.0, dtype=torch.float32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def within(got, want, bound):
    off = (got.double() - want).abs() - bound
    assert not bool(torch.isnan(off).any()) and bool((off <= 0).all()), float(off.max())


SHAPES = [(1, 8), (3, 64), (5, 512), (257, 520), (1030, 128), (2, 1024), (19, 1032), (700, 2048), (4, 2056), (1, 4096), (300, 4096), (2, 4104),
          (33, 8192), (1, 8200), (5, 16384)]


@pytest.mark.parametrize("x, stream", [("f32", None), ("bf16", None), ("f32", "bf16"), ("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("tokens, width", SHAPES)
def test_forward(nz, tokens, width, x, stream):
    eps = 1e-5
    x = normal(tokens, width, seed=1, std=0.5, dtype=TYPES[x])
    weight = 1 + normal(width, seed=2, std=0.2)
    residual = normal(tokens, width, seed=3, dtype=TYPES[stream]) if stream else None
    out = nz.neuzip_norm(x, weight, eps, residual)
    total = x
    if stream:
        y, total = out
        assert total.dtype == residual.dtype and torch.equal(total, (x.float() + residual.float()).to(residual.dtype))
    else:
        y = out
    s = total.double()
    want = s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt() * weight.double()
    within(y, want, want.abs() * (2.0 ** -8 + (width / 1024 + 20) * ULP) + 1e-37)
    if stream:      # in place, and into tensors of the caller's
        mine, there = residual.clone(), torch.empty_like(y)
        got = nz.neuzip_norm(x, weight, eps, mine, there, mine)
        assert got[0] is there and got[1] is mine and torch.equal(mine, total) and torch.equal(there, y)


@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("along", [False, True])
@pytest.mark.parametrize("tokens, width", SHAPES)
def test_backward(nz, tokens, width, along, stream):
    eps = 1e-5
    total = normal(tokens, width, seed=4, dtype=TYPES[stream])
    weight = 1 + normal(width, seed=5, std=0.2)
    grad_y = normal(tokens, width, seed=6, std=0.01, dtype=torch.bfloat16)
    grad_total = normal(tokens, width, seed=7, std=0.01, dtype=torch.bfloat16) if along else None
    grad_x, grad_weight = nz.neuzip_norm_backward(total, weight, grad_y, eps, grad_total)
    s, w, gy = total.double(), weight.double(), grad_y.double()
    n = 1 / (s.square().mean(dim=1, keepdim=True) + eps).sqrt()
    g = gy * w
    want = n * (g - s * n ** 2 * (g * s).mean(dim=1, keepdim=True))
    size = n * (g.abs() + s.abs() * n ** 2 * (g * s).abs().mean(dim=1, keepdim=True))
    if along:
        want, size = want + grad_total.double(), size + grad_total.double().abs()
    within(grad_x, want, want.abs() * 2.0 ** -8 + 3 * (width / 512 + 20) * ULP * size)
    terms = gy * s * n
    within(grad_weight, terms.sum(dim=0), (tokens + width / 1024 + 40) * ULP * terms.abs().sum(dim=0) + 1e-37)
    # one by one, in place, the same every time
    only, none = nz.neuzip_norm_backward(total, weight, grad_y, eps, grad_total, grad_weight=False)
    assert none is None and torch.equal(only, grad_x)
    none, only = nz.neuzip_norm_backward(total, weight, grad_y, eps, grad_total, grad_x=False)
    assert none is None and torch.equal(only, grad_weight)
    there = (grad_total if along else grad_y).clone()
    got, _ = nz.neuzip_norm_backward(total, weight, grad_y if along else there, eps, there if along else None, grad_x=there)
    assert got is there and torch.equal(there, grad_x)


@pytest.mark.parametrize("width", [24, 1160])
def test_gradients_against_differences(nz, width):
    """The formula of the backward pass, in 64 bits, against differences of the forward pass' formula; the kernel against the formula above."""
    tokens, eps, step = 3, 1e-2, 1e-5
    total, weight, grad_y = normal(tokens, width, seed=8), 1 + normal(width, seed=9, std=0.2), normal(tokens, width, seed=10, dtype=torch.bfloat16)
    grad_x, grad_weight = nz.neuzip_norm_backward(total, weight, grad_y, eps)

    def loss(s, w):
        return float((grad_y.double() * (s / (s.square().mean(dim=1, keepdim=True) + eps).sqrt() * w)).sum())

    s, w = total.double(), weight.double()
    for t, c in ((0, 0), (1, width // 2), (2, width - 1)):
        d = torch.zeros_like(s)
        d[t, c] = step
        want = (loss(s + d, w) - loss(s - d, w)) / (2 * step)
        # (a third derivative of some units times step^2, and the loss' own roundings over step)
        assert abs(float(grad_x[t, c]) - want) <= 2.0 ** -8 * abs(want) + 1e-5
        d = torch.zeros_like(w)
        d[c] = step
        want = (loss(s, w + d) - loss(s, w - d)) / (2 * step)
        assert abs(float(grad_weight[c]) - want) <= 1e-5 * (1 + abs(want))


@pytest.mark.parametrize("stream", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-15, 1e15])
def test_very_small_and_large_rows(nz, size, stream):
    """1 / rms to the third power is no binary32 number there, the gradients are."""
    tokens, width = 5, 264
    total = normal(tokens, width, seed=14, std=size, dtype=TYPES[stream])
    weight, grad_y = 1 + normal(width, seed=15, std=0.2), normal(tokens, width, seed=16, dtype=torch.bfloat16)
    s, w, gy = total.double(), weight.double(), grad_y.double()
    n = 1 / s.square().mean(dim=1, keepdim=True).sqrt()
    want = s * n * w
    within(nz.neuzip_norm(total, weight, 0.0), want, want.abs() * (2.0 ** -8 + (width / 1024 + 20) * ULP))
    grad_x, grad_weight = nz.neuzip_norm_backward(total, weight, grad_y, 0.0)
    g = gy * w
    want = n * (g - s * n ** 2 * (g * s).mean(dim=1, keepdim=True))
    within(grad_x, want, want.abs() * 2.0 ** -8 + 3 * (width / 512 + 20) * ULP * n * (g.abs() + s.abs() * n ** 2 * (g * s).abs().mean(dim=1, keepdim=True)))
    terms = gy * s * n
    within(grad_weight, terms.sum(dim=0), (tokens + width / 1024 + 40) * ULP * terms.abs().sum(dim=0))


def test_no_tokens(nz):
    weight = torch.ones(64, device=DEV)
    none = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    y, total = nz.neuzip_norm(none, weight, 1e-5, none)
    assert y.shape == total.shape == (0, 64)
    grad_x, grad_weight = nz.neuzip_norm_backward(none, weight, none, 1e-5)
    assert grad_x.shape == (0, 64) and bool((grad_weight == 0).all())


def test_rows_of_zeros_and_without_numbers(nz):
    """eps keeps a row of zeros finite; infinities and NaN stay in their row."""
    x = normal(5, 256, seed=11, dtype=torch.bfloat16)
    x[1] = 0
    x[2, 7] = float("inf")
    x[4, 0] = float("nan")
    weight = torch.ones(256, device=DEV)
    y = nz.neuzip_norm(x, weight, 1e-5)
    assert bool((y[1] == 0).all()) and bool(torch.isnan(y[4]).all()) and bool(torch.isnan(y[2, 7])) and bool((y[2, :7] == 0).all())
    for i in (0, 3):
        assert torch.equal(y[i], nz.neuzip_norm(x[i:i + 1].contiguous(), weight, 1e-5)[0])


def test_batch_by_sequence(nz):
    x, weight = normal(2, 5, 128, seed=12), torch.ones(128, device=DEV)
    residual = normal(2, 5, 128, seed=13, dtype=torch.bfloat16)
    y, total = nz.neuzip_norm(x, weight, 1e-5, residual)
    flat, _ = nz.neuzip_norm(x.view(10, 128), weight, 1e-5, residual.view(10, 128))
    assert y.shape == total.shape == (2, 5, 128) and torch.equal(y.view(10, 128), flat)
