// What stands in front of the linear layer's kernel: the outputs set up, the activations laid out.
#pragma once

#include "neuzip_format.h"

namespace nz {

constexpr uint32_t kLinMaxTokens = 64;   // of a tile
constexpr uint32_t kLinBatchMax = 4;     // weights of a launch

struct LinearInitArgs {
    float *y[kLinBatchMax];
    const float *bias[kLinBatchMax];
    uint32_t out_features[kLinBatchMax];
    uint32_t wg_end[kLinBatchMax];  // workgroups that set y up (none where the sums are stored whole) ...
    uint32_t set_up;                // ... of all weights
    const uint4 *x;                 // the activations, in pieces of 8 features, and where they go (nullptr: they stay)
    uint4 *scratch;
    uint32_t row_pieces;            // of a token
    uint32_t tokens;
};

// A workgroup of the launch in front, where there is something to do: y[t][o] = bias[o] (or 0), the accumulation target, four tokens of
// 256 outputs to a workgroup; and the activations in the order in which waves read them.
//
// A wave's operand is 32 or 64 bytes of each of 32 or 16 rows of x: as x lies, a request touches as many cache lines, and a CU
// of 16 waves is busy with these requests for longer than with the symbols (64 tokens, x as it lies / every request 1 KB in
// a piece: 4096 x 14336, k = 3, 65 / 47 us, 14336 x 4096 60 / 40, 4096 x 4096 27 / 18).  So, given the room, the tokens of 16
// neighbouring features are laid side by side, 32 bytes each (tile by tile of 64 tokens): whatever 16 or 32 of them a wave
// asks for are then neighbours.
constexpr uint32_t kLinInitThreads = 256, kLinInitTokens = 4;
__host__ __device__ constexpr uint32_t padded_tokens(uint32_t tokens) { return (tokens + 3) / 4 * 4; }  // 128 bytes
__device__ __forceinline__ void linear_init_workgroup(const LinearInitArgs &b, uint32_t wg)
{
    // which weight's y this workgroup sets up (a grid of outputs x tokens x weights, where this is known without a look at the ends
    // and without a division, gave nothing: 300 x 1152, 9 tokens, 17.7 us either way)
    float *y = nullptr;
    const float *bias = nullptr;
    uint32_t out_features = 1, first = 0;
#pragma unroll
    for (uint32_t i = 0; i < kLinBatchMax; ++i) {
        const uint32_t before = i ? b.wg_end[i - 1] : 0u;
        if (wg >= before && wg < b.wg_end[i]) {
            y = b.y[i];
            bias = b.bias[i];
            out_features = b.out_features[i];
            first = before;
        }
    }
    if (!y) {  // (behind them all)
        const uint64_t i = static_cast<uint64_t>(wg - b.set_up) * kLinInitThreads + threadIdx.x;
        if (i >= static_cast<uint64_t>(b.row_pieces) * b.tokens)
            return;
        // (neighbouring threads take neighbouring places: pieces 2p and 2p + 1 of one token behind those of the token before)
        const uint64_t tile_pieces = static_cast<uint64_t>(b.row_pieces) * kLinMaxTokens;
        const uint32_t tile = b.tokens > kLinMaxTokens ? static_cast<uint32_t>(i / tile_pieces) : 0u;
        const uint64_t in_tile = i - tile * tile_pieces;
        const uint32_t t0 = tile * kLinMaxTokens, tokens = min(b.tokens - t0, kLinMaxTokens), half = i & 1u;
        const uint32_t pair = static_cast<uint32_t>((in_tile >> 1) / tokens), token = static_cast<uint32_t>((in_tile >> 1) - static_cast<uint64_t>(pair) * tokens);
        uint4 *to = b.scratch + tile * tile_pieces;
        to[(static_cast<uint64_t>(pair) * padded_tokens(tokens) + token) * 2 + half] =
            b.x[static_cast<uint64_t>(t0 + token) * b.row_pieces + pair * 2 + half];
        return;
    }
    const uint32_t across = (out_features + kLinInitThreads - 1) / kLinInitThreads;
    const uint32_t o = (wg - first) % across * kLinInitThreads + threadIdx.x;
    const uint32_t t0 = (wg - first) / across * kLinInitTokens;
    if (o >= out_features)
        return;
    const float v = bias ? bias[o] : 0.0f;
#pragma unroll
    for (uint32_t t = t0; t < t0 + kLinInitTokens; ++t)
        if (t < b.tokens)
            y[static_cast<uint64_t>(t) * out_features + o] = v;
}

}  // namespace nz
