"""Forms of the operators' kernels that only larger calls take (-m gpu): the gradient's sort beside tables of more than 128 MB and of more
than 64 runs of 4096 tokens, the lookup of more than 8192 units with fewer mantissa bits and normalised, adapters beside a weight
without entry points.  Checks and bounds are those of test_gpu_embedding.py and test_gpu_adapters.py.
"""
import pytest
import torch

import test_gpu_adapters as adapted
import test_gpu_embedding as embedded
from paper_2410_20650_amd import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


# ------------------------------------------------------------------------------------------------ gradient
@pytest.mark.parametrize("count", [65, 4097, 9000])
def test_gradient_of_a_large_table(nz, count):
    rows, features = 33000, 2056
    assert rows * features // 8 > 1 << 23
    g = inputs.gaussian_bf16((count, features), 9100 + count, std=0.01, device=DEV)
    embedded.check_grad(nz, embedded.some_tokens(rows, count, count), g, rows, 0.3)     # (a fifth of the tokens are one row's)
    embedded.check_grad(nz, torch.full((count,), rows - 1, dtype=torch.int64, device=DEV), g, rows, 1.0)


@pytest.mark.parametrize("rows", [1000, 90000])
def test_gradient_of_more_than_64_runs(nz, rows):
    # 75 runs: rows of every run, of the first and the last, of late ones alone, of the 65th alone, of two neighbours among the late ones
    count, features = 75 * 4096 - 77, 8
    gen = torch.Generator().manual_seed(rows)
    tok = torch.randint(0, rows - 10, (count,), generator=gen)
    tok[torch.rand(count, generator=gen) < 0.1] = -1
    tok[::4096] = rows - 1
    tok[5], tok[count - 1] = rows - 2, rows - 2
    tok[66 * 4096 + 9::7777] = rows - 3
    tok[64 * 4096 + 17] = rows - 4
    tok[70 * 4096 + 100:71 * 4096 + 100] = rows - 5
    tok[3], tok[64 * 4096 + 3:64 * 4096 + 300], tok[70 * 4096 + 7] = rows - 6, rows - 6, rows - 6
    g = inputs.gaussian_bf16((count, features), 9150, std=0.01, device=DEV)
    embedded.check_grad(nz, tok.to(DEV), g, rows, 1.0)


# ------------------------------------------------------------------------------------------------ lookup
@pytest.mark.parametrize("rows,features", [(20000, 8), (700, 1160), (4099, 4096)])
@pytest.mark.parametrize("k", [3, 1, 0])
def test_many_tokens_with_fewer_mantissa_bits(nz, rows, features, k):
    w = inputs.gaussian_bf16((rows, features), 9200 + rows, device=DEV)
    blob = nz.neuzip_compress(w, k)
    embedded.check_lookup(nz, blob, embedded.kept(w, k), embedded.some_tokens(rows, 9001, 5), 1.0)
    embedded.check_lookup(nz, blob, embedded.kept(w, k), embedded.some_tokens(rows, 20000, 6), 22.627417)


@pytest.mark.parametrize("rows,features", [(600, 1160), (4099, 4096)])
@pytest.mark.parametrize("k,block", [(3, 32), (1, 512), (0, 128)])
def test_many_tokens_of_normalised_tables(nz, rows, features, k, block):
    w = inputs.student_t4_bf16((rows, features), 9300 + k, device=DEV)
    blob = nz.neuzip_compress_blockwise(w, k, block)
    table = torch.empty_like(w)
    nz.neuzip_decompress(blob, table)
    for scale in (1.0, 3.0):
        embedded.check_lookup(nz, blob, table, embedded.some_tokens(rows, 9001, k), scale)


@pytest.mark.parametrize("kind", ["random", "constant"])
def test_many_tokens_of_unusual_tables(nz, kind):
    # words that do not fit the window; a single exponent
    w = inputs.random_bits_bf16(1040 * 512, 9310, device=DEV).view(1040, 512) if kind == "random" else inputs.constant_bf16(1040 * 512, 0.125, device=DEV).view(1040, 512)
    embedded.check_lookup(nz, nz.neuzip_compress(w, 7), w, embedded.some_tokens(1040, 9001, 7), 1.0)


# ------------------------------------------------------------------------------------------------ adapters
# (more than 4096 chunks have no entry points: rows inside chunks, across them, longer than one)
@pytest.mark.parametrize("infeat,outfeat", [(640, 26500), (4096, 4100), (4736, 3551), (14336, 1180)])
@pytest.mark.parametrize("tokens", [1, 3, 9, 40, 64, 130])
def test_adapters_beside_a_weight_without_entry_points(nz, infeat, outfeat, tokens):
    assert infeat * outfeat > 4096 * 4096
    d = adapted.data(tokens, infeat, outfeat, 24, 7, 9400 + tokens)
    blob = nz.neuzip_compress(d["w"], 7)
    adapted.check(nz, d, blob, d["w"], d["bias"], d["scales"])
    adapted.check(nz, d, blob, d["w"])


@pytest.mark.parametrize("k,block", [(3, 0), (1, 0), (0, 0), (3, 128), (0, 512)])
def test_adapters_beside_a_lossy_weight_without_entry_points(nz, k, block):
    d = adapted.data(33, 4736, 3551, 16, 5, 9500 + k)
    blob = nz.neuzip_compress_blockwise(d["w"], k, block)
    kept = torch.empty_like(d["w"])
    nz.neuzip_decompress(blob, kept)
    adapted.check(nz, d, blob, kept, d["bias"], d["scales"])
