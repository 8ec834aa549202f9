"""The gated feed-forward block (-m gpu): from compressed weights, from decompressed ones, and its backward pass.

Products of bf16 words are exact and sums are binary32: a sum of n terms in any order is within n * 2^-24 of the sum of their
magnitudes.  sigmoid(z) = 1 / (1 + exp(-z)) is taken with the hardware's exponential and reciprocal: exp(-z) is 2^(-z log2 e), whose
argument is rounded (2^-24 of it) and doubles as a relative error of the power, and both instructions are good to a unit or two in the
last place, so 2^-20 + |z| * 2^-23 of the value is ample.  A result in bf16 has a rounding of 2^-8 at most on top of that.  The backward pass
rounds dg and du to bf16 (2^-8 each) before the matrix cores take them.
"""
import math

import numpy as np
import pytest
import torch

from paper_2410_20650_amd import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GUARD = 512
EPS, BF = 2.0 ** -24, 2.0 ** -8
C = 2 * math.sqrt(2 / math.pi)


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def guarded(shape, dtype=torch.bfloat16):
    """A tensor with GUARD elements on either side that nobody may touch."""
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * GUARD,), 7.0, dtype=dtype, device=DEV)
    return whole, whole[GUARD:GUARD + n].view(shape)


def untouched(*wholes):
    return all(bool((w[:GUARD] == 7.0).all()) and bool((w[-GUARD:] == 7.0).all()) for w in wholes)


def argument(g, act):
    return g if act == 0 else C * (g + 0.044715 * g ** 3)


def value(g, act):
    return g * torch.sigmoid(argument(g, act))


def slope(g, act):
    s = torch.sigmoid(argument(g, act))
    return s + g * s * (1 - s) * (1.0 if act == 0 else C * (1 + 0.134145 * g ** 2))


def steepest(g, off, act):
    """How much the activation can change when g is off by that much: its slope is below 1.13 everywhere."""
    return 1.13 * off


def wrong(act, g):
    """Relative error of a computed sigmoid."""
    return 2.0 ** -20 + argument(g, act).abs() * 2.0 ** -23


def check_h(h, g, u, g_size, u_size, act, terms):
    off_g, off_u = (terms + 64) * EPS * g_size, (terms + 64) * EPS * u_size
    want = value(g, act) * u
    bound = steepest(g, off_g, act) * (u.abs() + off_u) + value(g, act).abs() * off_u + want.abs() * (wrong(act, g) + 4 * EPS)
    bound = bound + BF * (want.abs() + bound) + 1e-30
    worst = float(((h.double() - want).abs() / bound).max())
    assert worst <= 1.0, worst


def products(x, wg, wu):
    x, wg, wu = x.double(), wg.double(), wu.double()
    return torch.matmul(x, wg.t()), torch.matmul(x, wu.t()), torch.matmul(x.abs(), wg.abs().t()), torch.matmul(x.abs(), wu.abs().t())


def data(tokens, infeat, outfeat, seed, std=0.02):
    return (inputs.gaussian_bf16((tokens, infeat), seed, std=1.0, device=DEV), inputs.gaussian_bf16((outfeat, infeat), seed + 1, std=std, device=DEV),
            inputs.gaussian_bf16((outfeat, infeat), seed + 2, std=std, device=DEV))


# ------------------------------------------------------------------------------------------------ from compressed weights
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("tokens", [1, 2, 9, 17, 33, 64, 65, 130])
@pytest.mark.parametrize("infeat,outfeat", [(128, 16), (384, 37), (4096, 200), (4736, 90)])
def test_serving_from_blobs(nz, infeat, outfeat, tokens, act):
    x, wg, wu = data(tokens, infeat, outfeat, 9000 + infeat + tokens, std=0.05)
    gate, up = nz.neuzip_compress(wg, 7), nz.neuzip_compress(wu, 7)
    whole, h = guarded((tokens, outfeat))
    nz.neuzip_gated_linear(gate, up, outfeat, infeat, x, act, h)
    nz.neuzip_check(gate)
    nz.neuzip_check(up)
    assert untouched(whole)
    check_h(h, *products(x, wg, wu), act, infeat)


@pytest.mark.parametrize("k,block", [(3, 0), (1, 0), (0, 0), (3, 128), (0, 512)])
def test_serving_from_lossy_blobs(nz, k, block):
    tokens, infeat, outfeat = 20, 1024, 120
    x, wg, wu = data(tokens, infeat, outfeat, 9100 + k, std=0.05)
    blobs = [nz.neuzip_compress_blockwise(w, k, block) for w in (wg, wu)]
    kept = [torch.empty_like(w) for w in (wg, wu)]
    nz.neuzip_decompress_batch(blobs, kept)
    h = nz.neuzip_gated_linear(*blobs, outfeat, infeat, x, nz.SILU)
    check_h(h, *products(x, *kept), 0, infeat)


def test_serving_on_a_stream_of_its_own_and_in_a_graph(nz):
    tokens, infeat, outfeat = 24, 4096, 512
    x, wg, wu = data(tokens, infeat, outfeat, 9150)
    first, second = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    gate, up = nz.neuzip_compress(wg, 7, stream=first), nz.neuzip_compress(wu, 7, stream=first)
    h = torch.empty((tokens, outfeat), dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    nz.neuzip_gated_linear(gate, up, outfeat, infeat, x, nz.SILU, h, stream=second)
    torch.cuda.synchronize()
    check_h(h, *products(x, wg, wu), 0, infeat)
    h2 = torch.empty_like(h)
    g2, u2 = (torch.empty((tokens, outfeat), device=DEV) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nz.neuzip_gated_linear(gate, up, outfeat, infeat, x, nz.SILU, h)
        nz.neuzip_gated_forward(x, wg, wu, nz.GELU_TANH, h2, keep=(g2, u2))
        grads = nz.neuzip_gated_backward(x, wg, wu, g2, u2, h, nz.GELU_TANH)
    for seed in (1, 2, 3):
        x.copy_(inputs.gaussian_bf16((tokens, infeat), 9160 + seed, std=1.0, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        check_h(h, *products(x, wg, wu), 0, infeat)
        eager = nz.neuzip_gated_forward(x, wg, wu, nz.GELU_TANH, keep=True)
        for one, other in zip((h2, g2, u2), eager):
            assert torch.equal(one, other)
        for one, other in zip(grads, nz.neuzip_gated_backward(x, wg, wu, g2, u2, h, nz.GELU_TANH)):
            assert torch.equal(one, other)


# ------------------------------------------------------------------------------------------------ from decompressed weights
# one token, tiles with ends of all kinds, depths that end inside a step, tiles of 256 and of 128 (several rounds of either), sums in slices
SHAPES = [(1, 8, 8), (3, 40, 16), (1, 1024, 512), (17, 200, 136), (64, 64, 64), (130, 264, 328), (257, 4096, 1032), (600, 72, 4104),
          (2000, 520, 2056), (33, 136, 9000), (1100, 1032, 9224), (5, 4104, 72)]


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("tokens,infeat,outfeat", SHAPES)
def test_forward(nz, tokens, infeat, outfeat, act):
    x, wg, wu = data(tokens, infeat, outfeat, 9200 + tokens, std=1.5 / math.sqrt(infeat))
    wholes, (h, gate, up) = zip(*[guarded((tokens, outfeat), dtype) for dtype in (torch.bfloat16, torch.float32, torch.float32)])
    nz.neuzip_gated_forward(x, wg, wu, act, h, keep=(gate, up))
    torch.cuda.synchronize()
    assert untouched(*wholes)
    g, u, g_size, u_size = products(x, wg, wu)
    check_h(h, g, u, g_size, u_size, act, infeat)
    for kept, want, size in ((gate, g, g_size), (up, u, u_size)):
        assert bool(((kept.double() - want).abs() <= (infeat + 64) * EPS * size + 1e-30).all())
    assert torch.equal(nz.neuzip_gated_forward(x, wg, wu, act), h)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("tokens,infeat,outfeat", SHAPES)
@pytest.mark.parametrize("alone", [False, True])
def test_backward(nz, tokens, infeat, outfeat, act, alone):
    x, wg, wu = data(tokens, infeat, outfeat, 9300 + tokens, std=1.5 / math.sqrt(infeat))
    gate, up = (inputs.gaussian_f32((tokens, outfeat), 9310 + i, std=1.5, device=DEV) for i in range(2))
    grad_h = inputs.gaussian_bf16((tokens, outfeat), 9320, std=0.1, device=DEV)
    whole_x, grad_x = guarded((tokens, infeat))
    whole_g, grad_g = guarded((outfeat, infeat))
    whole_u, grad_u = guarded((outfeat, infeat))

    def backward(grad_x, grad_g, grad_u):
        if not alone:
            return nz.neuzip_gated_backward(x, wg, wu, gate, up, grad_h, act, grad_x, (grad_g, grad_u) if grad_g is not None else True)
        (grad_x, _, _) = nz.neuzip_gated_backward(x, wg, wu, gate, up, grad_h, act, grad_x, False)
        (_, grad_g, grad_u) = nz.neuzip_gated_backward(x, wg, wu, gate, up, grad_h, act, False, (grad_g, grad_u) if grad_g is not None else True)
        return grad_x, grad_g, grad_u

    backward(grad_x, grad_g, grad_u)
    torch.cuda.synchronize()
    assert untouched(whole_x, whole_g, whole_u)
    g, u, gh = gate.double(), up.double(), grad_h.double()
    dg, du = gh * u * slope(g, act), gh * value(g, act)
    # the slope is a sum whose terms can cancel: off by the sigmoid's error of each of them
    s = torch.sigmoid(argument(g, act))
    terms = s + (g * s * (1 - s) * (1.0 if act == 0 else C * (1 + 0.134145 * g ** 2))).abs() + (g * s).abs() * (1.0 if act == 0 else C * (1 + 0.134145 * g ** 2))
    off_dg = (gh * u).abs() * terms * (wrong(act, g) + 8 * EPS)
    off_dg = off_dg + BF * (dg.abs() + off_dg)
    off_du = du.abs() * (wrong(act, g) + 8 * EPS)
    off_du = off_du + BF * (du.abs() + off_du)
    xs, gs, us = x.double(), wg.double(), wu.double()

    def check(got, want, off, size, n):
        bound = off + (n + 64) * EPS * (size + off)
        bound = bound + BF * (want.abs() + bound) + 1e-30
        worst = float(((got.double() - want).abs() / bound).max())
        assert worst <= 1.0, worst

    check(grad_x, torch.matmul(dg, gs) + torch.matmul(du, us), torch.matmul(off_dg, gs.abs()) + torch.matmul(off_du, us.abs()),
          torch.matmul(dg.abs(), gs.abs()) + torch.matmul(du.abs(), us.abs()), 2 * outfeat)
    check(grad_g, torch.matmul(dg.t(), xs), torch.matmul(off_dg.t(), xs.abs()), torch.matmul(dg.abs().t(), xs.abs()), tokens)
    check(grad_u, torch.matmul(du.t(), xs), torch.matmul(off_du.t(), xs.abs()), torch.matmul(du.abs().t(), xs.abs()), tokens)
    again = backward(True, None, None)
    for one, other in zip(again, (grad_x, grad_g, grad_u)):
        assert torch.equal(one, other)      # from run to run the same


def test_backward_of_what_is_wanted(nz):
    x, wg, wu = data(70, 136, 264, 9400)
    h, gate, up = nz.neuzip_gated_forward(x, wg, wu, keep=True)
    every = nz.neuzip_gated_backward(x, wg, wu, gate, up, h)
    only_x = nz.neuzip_gated_backward(x, wg, wu, gate, up, h, grad_weights=False)
    only_w = nz.neuzip_gated_backward(x, wg, wu, gate, up, h, grad_x=False)
    assert torch.equal(only_x[0], every[0]) and only_x[1:] == (None, None)
    assert only_w[0] is None and torch.equal(only_w[1], every[1]) and torch.equal(only_w[2], every[2])


def test_no_tokens(nz):
    x, wg, wu = data(1, 136, 264, 9410)
    none = torch.empty((0, 264), dtype=torch.bfloat16, device=DEV)
    h, gate, up = nz.neuzip_gated_forward(x[:0], wg, wu, keep=True)
    assert h.shape == (0, 264)
    grad_x, grad_g, grad_u = nz.neuzip_gated_backward(x[:0], wg, wu, gate, up, none)
    assert grad_x.shape == (0, 136) and not bool(grad_g.any()) and not bool(grad_u.any())


@pytest.mark.parametrize("act", [0, 1])
def test_large_and_infinite_values(nz, act):
    # weights that pick one input feature: g and u are what x holds
    n = 64
    x = torch.zeros((8, n), dtype=torch.bfloat16, device=DEV)
    x[0, :8] = torch.tensor([3e38, -3e38, 1e4, -1e4, 100.0, -100.0, 1e-38, -1e-38]).to(torch.bfloat16)
    eye = torch.eye(n, dtype=torch.bfloat16, device=DEV)
    ones = torch.zeros_like(eye)
    ones[:, n - 1] = 1.0
    x[:, n - 1] = 1.0       # (u = 1)
    h, gate, up = nz.neuzip_gated_forward(x, eye, ones, act, keep=True)
    assert torch.equal(gate, x.float()) and bool((up == 1).all())
    want = torch.where(x.double() > 50, x.double(), torch.where(x.double() < -50, torch.zeros_like(x.double()), value(x.double(), act)))
    assert bool(((h.double() - want).abs() <= BF * want.abs() * 1.01 + 1e-38).all())
    grad_h = torch.ones_like(h)
    grad_x, grad_g, grad_u = nz.neuzip_gated_backward(x, eye, ones, gate, up, grad_h, act, grad_weights=False)
    assert bool(torch.isfinite(grad_x[:, :n - 1]).all())
    assert bool((grad_x[0, :6].double() - torch.tensor([1.0, 0, 1, 0, 1, 0], dtype=torch.float64, device=DEV)).abs().max() <= BF)
    # an infinity or NaN in one token stays there
    x[3, 5], x[4, 5] = float("inf"), float("nan")
    h = nz.neuzip_gated_forward(x, eye, ones, act)
    bad = ~torch.isfinite(h).all(dim=1)
    assert bad.tolist() == [False, False, False, True, True, False, False, False]


@pytest.mark.parametrize("act", [0, 1])
def test_gradients_against_differences(nz, act):
    # the loss sum(h * r) in 64 bits, moved by a step in one entry of x or of a weight
    tokens, infeat, outfeat, step = 7, 24, 40, 1e-4
    x, wg, wu = data(tokens, infeat, outfeat, 9500, std=0.3)
    r = inputs.gaussian_bf16((tokens, outfeat), 9503, std=1.0, device=DEV)
    h, gate, up = nz.neuzip_gated_forward(x, wg, wu, act, keep=True)
    grads = nz.neuzip_gated_backward(x, wg, wu, gate, up, r, act)

    def loss(tensors):
        a, b, c = tensors
        return float((value(torch.matmul(a, b.t()), act) * torch.matmul(a, c.t()) * r.double()).sum())

    base = [t.double() for t in (x, wg, wu)]
    scale = [float(g.double().abs().max()) for g in grads]
    for which, (row, col) in ((0, (0, 0)), (0, (6, 23)), (1, (0, 5)), (1, (39, 23)), (2, (17, 3)), (2, (39, 0))):
        ends = []
        for sign in (1, -1):
            moved = [t.clone() for t in base]
            moved[which][row, col] += sign * step
            ends.append(loss(moved))
        difference = (ends[0] - ends[1]) / (2 * step)
        # (dg and du are bf16 words, and so is the gradient: each term of the sum is off by 2^-8 of itself, and the sum too)
        assert abs(difference - float(grads[which][row, col])) <= 6 * BF * scale[which]


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals(nz):
    x, wg, wu = data(5, 256, 64, 9600)
    gate, up = nz.neuzip_compress(wg, 7), nz.neuzip_compress(wu, 7)

    def code(call):
        with pytest.raises(nz.NeuzipError) as e:
            call()
        return e.value.code

    assert code(lambda: nz.neuzip_gated_linear(gate, up, 64, 256, x, 2)) == nz.EINVAL
    assert code(lambda: nz.neuzip_gated_linear(gate, up, 63, 256, x)) == nz.EINVAL
    assert code(lambda: nz.neuzip_gated_linear(gate, nz.neuzip_compress(wu, 3), 64, 256, x)) == nz.EINVAL
    assert code(lambda: nz.neuzip_gated_linear(gate, up, 64, 256, x[:0])) == nz.EINVAL
    assert code(lambda: nz.neuzip_gated_linear(gate, nz.neuzip_compress(wu.float(), 7), 64, 256, x)) == nz.EUNSUPPORTED
    assert code(lambda: nz.neuzip_gated_linear(gate, up, 64, 256, x, scratch=torch.empty(64, dtype=torch.uint8, device=DEV))) == nz.EINVAL
    with pytest.raises(ValueError):
        nz.neuzip_gated_linear(gate, up, 64, 257, x)
    assert code(lambda: nz.neuzip_gated_forward(x, wg, wu, 7)) == nz.EINVAL
    assert code(lambda: nz.neuzip_gated_forward(x[:, :252].contiguous(), wg[:, :252].contiguous(), wu[:, :252].contiguous())) == nz.EINVAL
    odd = torch.empty(64 * 256 + 8, dtype=torch.bfloat16, device=DEV)[1:1 + 64 * 256].view(64, 256)
    assert code(lambda: nz.neuzip_gated_forward(x, odd, wu)) == nz.EINVAL
    with pytest.raises(TypeError):
        nz.neuzip_gated_forward(x.float(), wg, wu)
    with pytest.raises(TypeError):
        nz.neuzip_gated_forward(x, wg, wu.t().contiguous().t())
    with pytest.raises(ValueError):
        nz.neuzip_gated_forward(x, wg, wu[:63])
    h, g, u = nz.neuzip_gated_forward(x, wg, wu, keep=True)
    with pytest.raises(ValueError):
        nz.neuzip_gated_backward(x, wg, wu, g[:4], u, h)
    with pytest.raises(TypeError):
        nz.neuzip_gated_backward(x, wg, wu, g, u, h.float())
    assert code(lambda: nz.neuzip_gated_backward(x, wg, wu, g, u, h, scratch=torch.empty(64, dtype=torch.uint8, device=DEV))) == nz.EINVAL
