"""A linear layer whose weight is held compressed, and the layer-by-layer training step of Alg. 1.

Orchestration only: every codec step is a call into the HIP library (binding.py); the dense
products of the backward pass are torch's (a library GEMM is the right tool for a training batch).

Alg. 1, forward loop: for each layer the weight is decompressed into temporary space just before
it is used (Sec. 2.2, Eq. (3)); here a decoding batch of up to 64 tokens goes through the fused
kernel instead, which never writes the weight.  Backward loop: the weight is decompressed again,
the gradients of the layer are formed, the optimiser step is applied at once and the weight is
compressed again, so that neither the uncompressed model nor the full set of gradients ever exists.

Biases are not compressed (Sec. 2.1 and 2.2 treat weight matrices only): they are plain float32
tensors of the caller's, and their addition and their own SGD step below are ordinary torch
arithmetic outside the codec's path.
"""
import torch

from . import binding as nz


class CompressedLinear:
    """y = x W^T + b with W (out_features x in_features, bf16) stored as a lossless blob."""

    def __init__(self, weight: torch.Tensor, bias: torch.Tensor = None, guard: int = 8):
        if weight.dim() != 2 or weight.dtype != torch.bfloat16:
            raise TypeError("weight: a 2-d bf16 tensor")
        self.out_features, self.in_features = weight.shape
        (self.blob,) = nz.neuzip_compress_guarded([weight.contiguous()], 7, guard)
        self.bias = None if bias is None else bias.to(torch.float32).contiguous()

    def weight_into(self, space: torch.Tensor) -> torch.Tensor:
        """W_hat <- decompress(c) into the caller's temporary space; returns it shaped as the matrix."""
        flat = space.view(-1)[: self.out_features * self.in_features]
        nz.neuzip_decompress(self.blob, flat)
        return flat.view(self.out_features, self.in_features)

    def forward(self, x: torch.Tensor, space: torch.Tensor) -> torch.Tensor:
        """x: tokens x in_features, bf16.  Returns float32 tokens x out_features."""
        tokens = x.shape[0]
        if tokens <= 64 and self.in_features % 128 == 0:
            return nz.neuzip_linear(self.blob, self.out_features, self.in_features, x.contiguous(), self.bias)
        y = torch.matmul(x, self.weight_into(space).t())
        # (the sum of a bf16 and a float32 tensor is float32, widening and addition in one launch, unless one of them has
        # no dimensions, which counts for less in torch's choice of the result's type)
        return y.float() if self.bias is None else y + torch.atleast_1d(self.bias)

    def backward_and_update(self, x: torch.Tensor, grad_y: torch.Tensor, lr: float, space: torch.Tensor,
                            grad_space: torch.Tensor):
        """The layer's part of the backward loop.  x: the input the forward pass saw (bf16), grad_y: the
        gradient of the loss with respect to the layer's output (bf16), both tokens x features.
        Returns (grad_x, rebuilt flag); the blob holds the updated weight afterwards and `grad_space`
        the weight gradient that was applied (bf16); what `space` holds is unspecified."""
        w_hat = self.weight_into(space)                                   # the second decompression
        grad_x = torch.matmul(grad_y, w_hat)                              # tokens x in_features
        n = self.out_features * self.in_features
        grad_w = grad_space.view(-1)[:n].view(self.out_features, self.in_features)
        torch.matmul(grad_y.t(), x, out=grad_w)                           # out_features x in_features, bf16
        if self.bias is not None:
            self.bias.sub_(grad_y.sum(dim=0, dtype=torch.float32), alpha=float(lr))
        # `space` still holds W_hat from the decompression above: the step and the coding are one pass,
        # and nobody needs the new weight uncompressed
        (rebuilt,) = nz.neuzip_update([self.blob], [grad_w.view(-1)], [space.view(-1)[:n]], lr, weights_ready=2)
        return grad_x, rebuilt


class CompressedEmbedding:
    """out[i] = scale * W[token[i]] with the table W (rows x features, bf16) stored as a lossless blob."""

    def __init__(self, table: torch.Tensor, scale: float = 1.0, guard: int = 8):
        if table.dim() != 2 or table.dtype != torch.bfloat16:
            raise TypeError("table: a 2-d bf16 tensor")
        self.rows, self.features = table.shape
        self.scale = float(scale)
        (self.blob,) = nz.neuzip_compress_guarded([table.contiguous()], 7, guard)

    def forward(self, tokens: torch.Tensor) -> torch.Tensor:
        """tokens: int64, any shape; -1 names no row.  Returns bf16, the rows decoded straight from the blob."""
        return nz.neuzip_embedding(self.blob, self.rows, self.features, tokens.contiguous(), self.scale)

    def backward_and_update(self, tokens: torch.Tensor, grad_out: torch.Tensor, lr: float, space: torch.Tensor,
                            grad_space: torch.Tensor):
        """The table's part of the backward loop: its gradient from grad_out (bf16), the step, compressed again.  `grad_space`
        holds the gradient afterwards; `space` is scratch memory of the table's size.  Returns the rebuilt flag."""
        n = self.rows * self.features
        grad = grad_space.view(-1)[:n]
        nz.neuzip_embedding_grad(tokens.contiguous(), grad_out.contiguous().view(-1, self.features), self.rows, self.scale, grad)
        (rebuilt,) = nz.neuzip_update([self.blob], [grad], [space.view(-1)[:n]], lr, weights_ready=3)
        return rebuilt


class CompressedGatedBlock:
    """h = act(x W_gate^T) * (x W_up^T), the first half of a gated feed-forward block, with both weights (out_features x
    in_features, bf16) stored as lossless blobs.  (The second half, the projection back, is a CompressedLinear.)"""

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, activation: int = nz.SILU, guard: int = 8):
        if w_gate.dim() != 2 or w_gate.dtype != torch.bfloat16 or w_up.dtype != torch.bfloat16 or w_up.shape != w_gate.shape:
            raise TypeError("weights: two 2-d bf16 tensors of one shape")
        self.out_features, self.in_features = w_gate.shape
        self.activation = activation
        self.blobs = nz.neuzip_compress_guarded([w_gate.contiguous(), w_up.contiguous()], 7, guard)

    def _pair(self, space: torch.Tensor):
        n = self.out_features * self.in_features
        room = (n + 7) // 8 * 8                                 # (both begin on 16 bytes)
        flat = space.view(-1)
        return [flat[at:at + n].view(self.out_features, self.in_features) for at in (0, room)]

    def weights_into(self, space: torch.Tensor):
        """Both weights decompressed into the caller's temporary space, in one launch."""
        pair = self._pair(space)
        nz.neuzip_decompress_batch(self.blobs, [w.view(-1) for w in pair])
        return pair

    def forward(self, x: torch.Tensor, space: torch.Tensor) -> torch.Tensor:
        """x: tokens x in_features, bf16 (batch x sequence for the tokens: the same).  Returns bf16 tokens x out_features.  space: room
        for both weights."""
        if 0 < x.numel() // self.in_features <= 64 and self.in_features % 128 == 0:     # (no tokens: nothing to serve)
            return nz.neuzip_gated_linear(*self.blobs, self.out_features, self.in_features, x.contiguous(), self.activation)
        return nz.neuzip_gated_forward(x.contiguous(), *self.weights_into(space), self.activation)

    def backward_and_update(self, x: torch.Tensor, grad_h: torch.Tensor, lr: float, space: torch.Tensor, grad_space: torch.Tensor):
        """The block's part of the backward loop.  The weights are decompressed a second time and the two products formed anew
        from the block's input (activation checkpointing), so that neither is kept from the forward pass.  Returns (grad_x,
        rebuilt flags); `grad_space` holds the two gradients that were applied, one behind the other."""
        x, grad_h = x.contiguous(), grad_h.contiguous()
        weights, grads = self.weights_into(space), self._pair(grad_space)
        _, gate, up = nz.neuzip_gated_forward(x, *weights, self.activation, keep=True)
        grad_x, _, _ = nz.neuzip_gated_backward(x, *weights, gate, up, grad_h, self.activation, grad_weights=grads)
        rebuilt = nz.neuzip_update(self.blobs, [g.view(-1) for g in grads], [w.view(-1) for w in weights], lr, weights_ready=2)
        return grad_x, rebuilt


class AdaptedLinear:
    """A CompressedLinear that serves several fine-tuned variants at once: beside the shared weight, adapter i is
    scales[i] * B[i] A[i], with A (adapters x rank x in_features) and B (adapters x out_features x rank) in bf16."""

    def __init__(self, base: CompressedLinear, a: torch.Tensor, b: torch.Tensor, scales: torch.Tensor = None):
        self.base, self.a, self.b = base, a.contiguous(), b.contiguous()
        self.scales = None if scales is None else scales.to(torch.float32).contiguous()

    def forward(self, x: torch.Tensor, ids: torch.Tensor) -> torch.Tensor:
        """x: tokens x in_features, bf16; ids: each token's adapter, int32, -1 for none.  Returns float32."""
        base = self.base
        return nz.neuzip_linear_adapters(base.blob, base.out_features, base.in_features, x.contiguous(), self.a, self.b, self.scales,
                                         ids, base.bias)


class ResidualNorm:
    """What stands between two layers: stream <- stream + x, y = stream / rms(stream) * weight.  The weight is not compressed: float32, as the biases."""

    def __init__(self, weight: torch.Tensor, eps: float = 1e-5):
        self.weight, self.eps = weight.to(torch.float32).contiguous(), float(eps)

    def forward(self, x: torch.Tensor, stream: torch.Tensor = None):
        """x: a layer's result (bf16 or float32) and the stream it is added to, in whose type the sum is held; without a stream x is the stream.
        Returns (y, stream), y in bf16."""
        if stream is None:
            return nz.neuzip_norm(x.contiguous(), self.weight, self.eps), x
        return nz.neuzip_norm(x.contiguous(), self.weight, self.eps, stream.contiguous())

    def backward_and_update(self, stream: torch.Tensor, grad_y: torch.Tensor, grad_stream: torch.Tensor, lr: float):
        """The norm's part of the backward loop.  stream: as forward returned it; grad_stream: the gradient that comes back along it (bf16), or None.
        Returns the gradient of the stream before and of x, which is one (bf16); the weight has made its step."""
        if grad_stream is not None:
            grad_stream = grad_stream.contiguous()
        grad_x, grad_weight = nz.neuzip_norm_backward(stream.contiguous(), self.weight, grad_y.contiguous(), self.eps, grad_stream)
        self.weight.sub_(grad_weight, alpha=float(lr))
        return grad_x


class CompressedAttention:
    """The attention block of a served model: the projections to queries, keys and values and back, all four stored as lossless blobs, around a cache that
    holds the keys and values of the tokens so far in 8 bits."""

    def __init__(self, w_q: torch.Tensor, w_k: torch.Tensor, w_v: torch.Tensor, w_o: torch.Tensor, head_dim: int, rotary: torch.Tensor = None,
                 window: int = 0, guard: int = 8):
        self.queries, self.keys, self.values, self.out = (CompressedLinear(w, guard=guard) for w in (w_q, w_k, w_v, w_o))
        self.head_dim, self.heads, self.window = head_dim, w_k.shape[0] // head_dim, int(window)
        if (w_k.shape != w_v.shape or w_q.shape[1] != w_k.shape[1] or w_k.shape[0] % head_dim or self.heads == 0 or w_q.shape[0] % w_k.shape[0]
                or w_o.shape[1] != w_q.shape[0]):
            raise ValueError("projections to query heads, as many or several to each head of the keys and values, and back")
        self.rotary = None if rotary is None else rotary.to(torch.float32).contiguous()

    def new_cache(self, pages: int, page_tokens: int = 64, device="cuda") -> nz.KeyValueCache:
        return nz.KeyValueCache.empty(pages, self.heads, self.head_dim, page_tokens, device)

    def forward(self, x: torch.Tensor, cache: nz.KeyValueCache, sequences: nz.Sequences, space: torch.Tensor, longest: int = 0) -> torch.Tensor:
        """x: rows x in_features, bf16, the newest tokens of the sequences, whose lengths count them already.  They are put into the cache and look back at
        it.  Returns float32 rows x out_features.  longest: no sequence has more tokens; without it the attention's form is chosen for sequences that
        fill their rows of the table, which costs time and scratch memory where a table has much more room than they have tokens (the attention of a prompt of 512
        tokens, 32 heads on 8 of 128, in a table for 131072: 37 us and 34 MB for 12 us and none; of 2048: 69 us for 59)."""
        if x.shape[0] == 0:
            return torch.empty((0, self.out.out_features), dtype=torch.float32, device=x.device)
        parts = (self.queries, self.keys, self.values)
        if x.shape[0] <= 64 and self.queries.in_features % 128 == 0:     # (one launch for the three)
            q, k, v = nz.neuzip_linear_batch([p.blob for p in parts], [p.out_features for p in parts], self.queries.in_features, x.contiguous())
        else:
            q, k, v = (p.forward(x, space) for p in parts)
        turned = nz.neuzip_cache_append(cache, sequences, k, v, q, self.rotary)
        seen = nz.neuzip_cache_attention(cache, sequences, turned, window=self.window, longest=longest)
        return self.out.forward(seen.view(x.shape[0], self.out.in_features), space)


def training_step(layers, x: torch.Tensor, target: torch.Tensor, lr: float, space: torch.Tensor,
                  grad_space: torch.Tensor, observer=None):
    """One step of Alg. 1 on a stack of CompressedLinear layers with ReLU between them and a squared
    error loss: forward layer by layer keeping the layer inputs, then backward in reverse order, each
    weight updated and recompressed as soon as its gradient exists.  Returns (loss, rebuilt flags).
    observer(i, layer_input, grad_y, grad_w), if given, is called right after layer i's update."""
    inputs, h = [], x
    for i, layer in enumerate(layers):
        inputs.append(h)
        y = layer.forward(h, space)
        h = (torch.relu(y) if i + 1 < len(layers) else y).to(torch.bfloat16)
    diff = h.float() - target.float()
    loss = 0.5 * (diff * diff).sum().item()
    grad = diff.to(torch.bfloat16)
    flags = [0] * len(layers)
    for i in reversed(range(len(layers))):
        if i + 1 < len(layers):
            grad = grad * (inputs[i + 1] > 0)                            # ReLU of layer i fed layer i + 1
        grad_y = grad.contiguous()
        grad, flags[i] = layers[i].backward_and_update(inputs[i], grad_y, lr, space, grad_space)
        if observer is not None:
            n = layers[i].out_features * layers[i].in_features
            observer(i, inputs[i], grad_y, grad_space.view(-1)[:n].view(layers[i].out_features, layers[i].in_features))
    return loss, flags
