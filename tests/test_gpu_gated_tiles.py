"""The gated feed-forward block in tiles of 256, with ragged ends of everything, and in what goes with them (-m gpu): sums in slices, gradients
in a launch each.  Checks and bounds are those of test_gpu_gated.py; test_gated_forms.py asks the library's rule which forms these shapes take.
"""
import pytest

import test_gpu_gated as blocks

pytestmark = pytest.mark.gpu

# tokens, in_features, out_features: last tiles of one token or of eight features, last steps of one token or of eight features
SHAPES = [(513, 2056, 10248), (1281, 1032, 9224), (401, 5384, 8200), (137, 7176, 10248), (2049, 4104, 1544), (1985, 2824, 8456), (1000, 4104, 14344),
          (1000, 4096, 14336)]


@pytest.fixture(scope="module")
def nz():
    from paper_2410_20650_amd import binding
    return binding


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("tokens,infeat,outfeat", SHAPES)
def test_forward(nz, tokens, infeat, outfeat, act):
    blocks.test_forward(nz, tokens, infeat, outfeat, act)


@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("tokens,infeat,outfeat", SHAPES)
def test_backward(nz, tokens, infeat, outfeat, act, alone):
    blocks.test_backward(nz, tokens, infeat, outfeat, act, alone)
