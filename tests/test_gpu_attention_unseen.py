"""Keys that a token does not see have no influence on it (-m gpu): later tokens' keys that take all the weight of those who see them leave the earlier tokens' rows
as they are, bit for bit, also where both are rows of one workgroup.
"""
import pytest
import torch

from cache_reference import E4M3
from test_gpu_cache import ints

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
# heads, group, head_dim, page, (new tokens, tokens with them), the new token whose key is the large one
CASES = {
    "few, four waves": (64, 2, 64, 64, [(3, 3000)] * 8, 2),
    "few, eight waves": (2, 4, 128, 64, [(3, 1900)] * 4, 2),
    "few, short pages": (2, 4, 128, 16, [(3, 1900)] * 4, 1),
    "some": (2, 4, 64, 64, [(40, 1100)] * 4, 35),
    "some, 128": (2, 4, 128, 32, [(40, 1100)] * 4, 3),
    "many": (8, 4, 128, 16, [(200, 1000)] * 4, 130),
    "many, 64": (8, 4, 64, 64, [(1500, 2200), (700, 900)], 650),
    "most": (8, 4, 128, 64, [(900, 9000)], 645),
}


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


def normal(*shape, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV)


@pytest.mark.parametrize("case", CASES)
def test_rows_before_a_large_key(nz, case):
    heads, group, dim, page, plan, large = CASES[case]
    wide = max((length + page - 1) // page for _, length in plan)
    table = torch.arange(len(plan) * wide, dtype=torch.int32, device=DEV).view(len(plan), wide)
    cache = nz.KeyValueCache(normal(len(plan) * wide, heads, page, dim, seed=1).clamp(-6, 6).to(E4M3), normal(len(plan) * wide, heads, dim, page, seed=2).to(E4M3),
                             *(torch.ones((len(plan) * wide, heads), device=DEV) for _ in range(2)))
    starts = [0]
    for n, _ in plan:
        starts.append(starts[-1] + n)
    q = normal(starts[-1], heads * group, dim, seed=3).abs().to(torch.bfloat16)
    sequences = nz.Sequences(ints(starts), ints([length for _, length in plan]), table)
    before = nz.neuzip_cache_attention(cache, sequences, q)
    again = nz.neuzip_cache_attention(cache, sequences, q)
    assert torch.equal(before, again)
    earlier = torch.zeros(starts[-1], dtype=torch.bool, device=DEV)
    for s, (n, length) in enumerate(plan):
        at = length - n + large
        cache.k.view(torch.uint8)[s * wide + at // page, :, at % page] = 0x58       # 16 in every feature: all queries' products with it are far above the others
        earlier[starts[s]:starts[s] + large] = True
    got = nz.neuzip_cache_attention(cache, sequences, q)
    assert torch.equal(got[earlier], before[earlier])
    assert not torch.equal(got[~earlier], before[~earlier])
