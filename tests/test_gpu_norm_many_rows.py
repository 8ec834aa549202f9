"""The norm of rows of more than 8192 elements, 1024 threads to a row, of so many tokens that their threads pass 32 bits (-m gpu): every row once, the first, the last and
those around the 2^22nd by themselves.  (140 or 210 GB of the device's memory.)
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF = torch.bfloat16
WIDTH, EPS, BEYOND = 8200, 1e-5, 1 << 22
TOKENS = BEYOND + 7


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    yield binding
    torch.cuda.empty_cache()


def normal(*shape, seed, dtype=BF):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


@pytest.mark.parametrize("stream", [False, True])
def test_tokens_whose_threads_pass_32_bits(nz, stream):
    torch.cuda.empty_cache()
    need = (3 if stream else 2) * TOKENS * WIDTH * 2
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip("not so much of the device's memory is free")
    weight = normal(WIDTH, seed=1, dtype=torch.float32)
    usual, apart = normal(1, WIDTH, seed=2), normal(9, WIDTH, seed=3)
    at = torch.tensor([0, 1, BEYOND - 3, BEYOND - 2, BEYOND - 1, BEYOND, BEYOND + 1, TOKENS - 2, TOKENS - 1], device=DEV)
    x = usual.expand(TOKENS, WIDTH).contiguous()
    x[at] = apart
    y = torch.full((TOKENS, WIDTH), 7.0, dtype=BF, device=DEV)
    residual = total = held = None
    if stream:
        residual = torch.ones((TOKENS, WIDTH), dtype=BF, device=DEV)
        ones, total, held = residual[:9].clone(), residual, (usual + 1, apart + 1)
    nz.neuzip_norm(x, weight, EPS, residual, y, total)
    for rows, got, summed in ((apart, y[at], 1), (usual, y[5:6], 0)):
        want = nz.neuzip_norm(rows, weight, EPS, ones[:rows.shape[0]] if stream else None)
        assert torch.equal(got, want[0] if stream else want)
        assert not stream or torch.equal(total[at] if summed else total[5:6], held[summed])
    for tensor in (y, total) if stream else (y,):       # (in pieces: what equal() makes is as large)
        every = tensor[5:6].clone()
        tensor[at] = every
        for piece in tensor.split(1 << 18):
            assert bool((piece == every).all())
