"""A small model whose weights are all held compressed: an embedding, a gated feed-forward block with its projection back, and an
output projection.  Trained layer by layer as Alg. 1 has it, then served token by token with the adapters of several requests.

    python -m paper_2410_20650_amd.small_model [--steps 8] [--tokens 512]

prints the loss of every step, what the weights take, and how the served outputs differ from the trained model's.
"""
import argparse

import torch

from . import binding as nz
from . import inputs
from .layer import AdaptedLinear, CompressedEmbedding, CompressedGatedBlock, CompressedLinear


class SmallModel:
    """y = W_out (h + W_down (act(W_gate h) * W_up h)) with h = scale * embedding[token]."""

    def __init__(self, rows=2000, width=256, hidden=640, classes=128, activation=nz.SILU, seed=1, device="cuda:0"):
        def weight(shape, tag, std):
            return inputs.gaussian_bf16(shape, seed * 100 + tag, std=std, device=device)

        self.embedding = CompressedEmbedding(weight((rows, width), 0, 0.02), scale=width ** 0.5)
        self.block = CompressedGatedBlock(weight((hidden, width), 1, width ** -0.5), weight((hidden, width), 2, width ** -0.5), activation)
        self.down = CompressedLinear(weight((width, hidden), 3, hidden ** -0.5))
        self.out = CompressedLinear(weight((classes, width), 4, width ** -0.5))
        most = max(rows * width, 2 * ((hidden * width + 7) // 8 * 8), classes * width)
        # one temporary space for whatever weight is in use, and one for its gradient
        self.space = torch.zeros(most, dtype=torch.bfloat16, device=device)
        self.grad_space = torch.zeros_like(self.space)

    def blobs(self):
        return [self.embedding.blob, *self.block.blobs, self.down.blob, self.out.blob]

    def forward(self, tokens):
        """Returns (y, the inputs of the layers)."""
        h = self.embedding.forward(tokens)
        gated = self.block.forward(h, self.space)
        mixed = (h.float() + self.down.forward(gated, self.space)).to(torch.bfloat16)
        return self.out.forward(mixed, self.space), (h, gated, mixed)

    def training_step(self, tokens, target, lr):
        """Squared error against target; every weight is stepped and compressed again as soon as its gradient exists.  Returns
        the loss."""
        y, (h, gated, mixed) = self.forward(tokens)
        diff = y.float() - target.float()
        loss = 0.5 * float((diff * diff).sum()) / tokens.numel()
        grad = (diff / tokens.numel()).to(torch.bfloat16)
        grad, _ = self.out.backward_and_update(mixed, grad, lr, self.space, self.grad_space)
        grad_gated, _ = self.down.backward_and_update(gated, grad.contiguous(), lr, self.space, self.grad_space)
        grad_h, _ = self.block.backward_and_update(h, grad_gated, lr, self.space, self.grad_space)
        self.embedding.backward_and_update(tokens, (grad.float() + grad_h.float()).to(torch.bfloat16), lr, self.space, self.grad_space)
        return loss

    def serve(self, tokens, adapted: AdaptedLinear, ids):
        """The outputs of single tokens of many requests, the output projection with each request's adapter."""
        h = self.embedding.forward(tokens)
        mixed = (h.float() + self.down.forward(self.block.forward(h, self.space), self.space)).to(torch.bfloat16)
        return adapted.forward(mixed, ids)


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=8)
    parser.add_argument("--tokens", type=int, default=512)
    args = parser.parse_args(argv)
    device = "cuda:0"
    model = SmallModel(device=device)
    generator = torch.Generator(device=device)
    generator.manual_seed(7)
    tokens = torch.randint(0, model.embedding.rows, (args.tokens,), generator=generator, device=device)
    target = inputs.gaussian_bf16((args.tokens, model.out.out_features), 11, std=1.0, device=device)
    losses = []
    for step in range(args.steps):
        losses.append(model.training_step(tokens, target, 0.05))
        print(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    held = sum(b.compressed_bytes for b in model.blobs())
    plain = 2 * sum(b.elems for b in model.blobs())
    print(f"weights: {held} bytes, {held / plain:.3f} of bf16", flush=True)
    # a decoding batch: one token each of many requests, some with an adapter
    batch, rank, adapters = 24, 16, 4
    a = inputs.gaussian_bf16((adapters, rank, model.out.in_features), 12, std=model.out.in_features ** -0.5, device=device)
    b = inputs.gaussian_bf16((adapters, model.out.out_features, rank), 13, std=0.1, device=device)
    ids = (torch.arange(batch, device=device) % (adapters + 1) - 1).to(torch.int32)
    served = model.serve(tokens[:batch], AdaptedLinear(model.out, a, b), ids)
    alone, _ = model.forward(tokens[:batch])
    apart = (served - alone).abs().amax(dim=1)
    print(f"served: {int((ids < 0).sum())} tokens without an adapter differ by at most {float(apart[ids < 0].max()):.1e}, "
          f"the others by {float(apart[ids >= 0].mean()):.3f} on average", flush=True)
    for blob in model.blobs():
        nz.neuzip_check(blob)
    return losses


if __name__ == "__main__":
    main()
