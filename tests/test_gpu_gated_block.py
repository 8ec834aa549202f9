"""CompressedGatedBlock on inputs of every number of tokens (-m gpu)."""
import pytest
import torch

from paper_2410_20650_amd import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("infeat", [256, 264])
def test_no_tokens(infeat):
    from paper_2410_20650_amd.layer import CompressedGatedBlock
    w_gate, w_up = (inputs.gaussian_bf16((40, infeat), 9900 + i, device=DEV) for i in range(2))
    block = CompressedGatedBlock(w_gate, w_up)
    space, grad_space = (torch.zeros(2 * 40 * infeat, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    x = torch.empty((0, infeat), dtype=torch.bfloat16, device=DEV)
    h = block.forward(x, space)
    assert h.shape == (0, 40)
    grad_x, _ = block.backward_and_update(x, h, 0.5, space, grad_space)
    assert grad_x.shape == (0, infeat) and not bool(grad_space.any())
    for held, w in zip(block.weights_into(space), (w_gate, w_up)):
        assert torch.equal(held, w)


def test_batch_and_sequence():
    from paper_2410_20650_amd.layer import CompressedGatedBlock
    block = CompressedGatedBlock(*(inputs.gaussian_bf16((40, 256), 9910 + i, std=0.06, device=DEV) for i in range(2)))
    space = torch.zeros(2 * 40 * 256, dtype=torch.bfloat16, device=DEV)
    x = inputs.gaussian_bf16((3, 50, 256), 9912, std=1.0, device=DEV)
    assert torch.equal(block.forward(x, space), block.forward(x.view(150, 256), space))
