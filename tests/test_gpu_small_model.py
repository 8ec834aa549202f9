"""The model of compressed weights that the operators make up together (-m gpu): its step against plain arithmetic on the same
weights, its loss, and single tokens served with adapters.
"""
import pytest
import torch

from paper_2410_20650_amd import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def held(blob, shape):
    from paper_2410_20650_amd import binding as nz
    w = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    nz.neuzip_decompress(blob, w)
    return w


def weights(model):
    e, g, d, o = model.embedding, model.block, model.down, model.out
    return [held(b, s) for b, s in ((e.blob, (e.rows, e.features)), (g.blobs[0], (g.out_features, g.in_features)),
                                    (g.blobs[1], (g.out_features, g.in_features)), (d.blob, (d.out_features, d.in_features)),
                                    (o.blob, (o.out_features, o.in_features)))]


def plain_loss(ws, scale, tokens, target):
    """The model in 64 bits, differentiated by torch on the CPU."""
    table, gate, up, down, out = ws
    h = scale * table[tokens]
    a, b = h @ gate.t(), h @ up.t()
    y = (h + (a * torch.sigmoid(a) * b) @ down.t()) @ out.t()
    return 0.5 * ((y - target) ** 2).sum() / tokens.numel()


@pytest.mark.parametrize("tokens", [40, 300])
def test_a_step_is_the_plain_one(tokens):
    # (40: the layers take their weights from the blobs; 300: from temporary space)
    from paper_2410_20650_amd.small_model import SmallModel
    model = SmallModel(rows=500)
    before = weights(model)
    g = torch.Generator().manual_seed(3)
    tok = torch.randint(0, 500, (tokens,), generator=g).to(DEV)
    target = inputs.gaussian_bf16((tokens, 128), 21, std=1.0, device=DEV)
    lr = 8.0
    loss = model.training_step(tok, target, lr)
    leaves = [w.double().cpu().requires_grad_() for w in before]
    want = plain_loss(leaves, model.embedding.scale, tok.cpu(), target.double().cpu())
    want.backward()
    assert abs(loss - float(want.detach())) <= 0.02 * float(want.detach())
    for leaf, old, new in zip(leaves, before, weights(model)):
        moved, right = (old.double() - new.double()).cpu(), lr * leaf.grad
        # bf16 words all along the way (activations, gradients) and the new weight rounded to bf16: in the mean a few per cent of the step,
        # and no entry further off than its weight's rounding and a tenth of the largest step
        assert float((moved - right).norm()) <= 0.05 * float(right.norm()) + 2.0 ** -8 * float(new.double().norm())
        assert bool(((moved - right).abs() <= 2.0 ** -8 * new.double().cpu().abs() + 0.1 * right.abs().max()).all())


def test_the_loss_falls_and_adapters_serve(capsys):
    from paper_2410_20650_amd import small_model
    losses = small_model.main(["--steps", "6", "--tokens", "200"])
    assert losses[-1] < 0.9 * losses[0]
    assert "served" in capsys.readouterr().out


def test_served_tokens_are_the_definition():
    from paper_2410_20650_amd.layer import AdaptedLinear
    from paper_2410_20650_amd.small_model import SmallModel
    model = SmallModel(rows=300)
    tok = torch.arange(10, device=DEV) * 7
    a = inputs.gaussian_bf16((3, 8, 256), 31, std=0.06, device=DEV)
    b = inputs.gaussian_bf16((3, 128, 8), 32, std=0.3, device=DEV)
    ids = (torch.arange(10, device=DEV) % 4 - 1).to(torch.int32)
    y = model.serve(tok, AdaptedLinear(model.out, a, b, torch.tensor([0.5, 1.0, 2.0], device=DEV)), ids)
    _, (_, _, mixed) = model.forward(tok)
    want = mixed.double() @ weights(model)[-1].double().t()
    for t in range(10):
        i = int(ids[t])
        if i >= 0:
            want[t] += [0.5, 1.0, 2.0][i] * (b[i].double() @ (a[i].double() @ mixed[t].double()))
    assert bool(((y.double() - want).abs() <= 1e-4 * (1 + want.abs())).all())


def test_layers_refuse_what_they_cannot_hold():
    from paper_2410_20650_amd.layer import CompressedEmbedding, CompressedGatedBlock
    w = inputs.gaussian_bf16((64, 256), 40, device=DEV)
    with pytest.raises(TypeError):
        CompressedEmbedding(w.float())
    with pytest.raises(TypeError):
        CompressedGatedBlock(w, w[:32])
