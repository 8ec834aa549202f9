// Penalties, biases and masks on logits for gfx950.
//
// One pass over the logits, a slice of a row's tokens to a workgroup.  The workgroup first counts, in LDS, how often each token of its slice
// occurs in the row's history, and finds the last bias entry of each; both with integer atomics, whose order does not show.  Every workgroup of a
// row reads the whole history (8 bytes a token, from the second one on out of a cache), which is why a slice is not shorter than it has to be for
// all CUs to have one.  What bounds it: reading and writing the logits once; for one row, the launch and the history's way through the caches.
// Measured, 128256 tokens: 48 rows with up to 4000 tokens of history 15.3 us (57 MB, 3.7 TB/s: a third of the workgroups start when the others have ended, and
// first read their history), one row with 1000 3.4 us.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace nz {

struct LogitsArgs {
    const float *logits;
    float *out;
    const int64_t *history;
    const int32_t *history_starts;
    const float *repetition, *frequency, *presence;
    const int64_t *bias_tokens;
    const float *bias_values;
    const int32_t *bias_starts;
    const int32_t *masks, *mask_ids;
    uint64_t history_tokens, bias_entries;
    uint64_t mask_words;
    uint32_t mask_count;
    uint32_t vocab;
};

struct LogitsRange {
    uint64_t begin, end;
};

// [starts[row], starts[row + 1]), inside 0 .. most
__device__ __forceinline__ LogitsRange logits_range(const int32_t *starts, uint32_t row, uint64_t most)
{
    const int32_t a = starts[row], b = starts[row + 1];
    LogitsRange r;
    r.begin = a < 0 ? 0 : static_cast<uint64_t>(a);
    r.end = b < 0 ? 0 : static_cast<uint64_t>(b);
    r.end = r.end < most ? r.end : most;
    return r;
}

// f(i) for i = threadIdx.x, + THREADS, ... below count, the loads of four of them on their way together
template <uint32_t THREADS, class F>
__device__ __forceinline__ void logits_each(const int64_t *tokens, uint64_t begin, uint64_t end, const F &f)
{
    for (uint64_t at = begin + threadIdx.x; at < end; at += 4 * THREADS) {
        int64_t token[4];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            token[j] = at + j * THREADS < end ? tokens[at + j * THREADS] : -1;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            f(at + j * THREADS, token[j]);
    }
}

// WIDE: rows begin on 16 bytes, a lane has four tokens side by side; else they are THREADS apart.
template <uint32_t SLICE, uint32_t THREADS, bool WIDE>
__global__ void __launch_bounds__(THREADS) logits_kernel(const LogitsArgs a)
{
#pragma clang fp contract(off)
    constexpr uint32_t kQuads = SLICE / THREADS / 4;
    __shared__ __align__(16) uint32_t counts[SLICE], entries[SLICE];  // entries: one more than the last entry's number in the row, 0: none
    const uint32_t row = blockIdx.y, first = blockIdx.x * SLICE;
    const uint32_t wide = a.vocab - first < SLICE ? a.vocab - first : SLICE;
    const uint64_t at = static_cast<uint64_t>(row) * a.vocab + first;
    const auto place = [&](uint32_t quad, uint32_t c) { return WIDE ? (quad * THREADS + threadIdx.x) * 4 + c : (quad * 4 + c) * THREADS + threadIdx.x; };
    // (on their way while the history is counted)
    float x[kQuads][4];
#pragma unroll
    for (uint32_t quad = 0; quad < kQuads; ++quad) {
        if constexpr (WIDE) {
            if (place(quad, 0) < wide) {
                const float4 v = *reinterpret_cast<const float4 *>(a.logits + at + place(quad, 0));
                x[quad][0] = v.x, x[quad][1] = v.y, x[quad][2] = v.z, x[quad][3] = v.w;
            }
        } else {
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c)
                if (place(quad, c) < wide)
                    x[quad][c] = a.logits[at + place(quad, c)];
        }
    }
    for (uint32_t i = threadIdx.x * 4; i < SLICE; i += THREADS * 4) {
        *reinterpret_cast<uint4 *>(counts + i) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(entries + i) = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    LogitsRange named = {0, 0};
    if (a.history) {
        const LogitsRange r = logits_range(a.history_starts, row, a.history_tokens);
        logits_each<THREADS>(a.history, r.begin, r.end, [&](uint64_t, int64_t token) {
            const uint64_t slot = static_cast<uint64_t>(token) - first;
            if (token >= 0 && slot < wide)
                atomicAdd(&counts[slot], 1u);
        });
    }
    if (a.bias_tokens) {
        named = logits_range(a.bias_starts, row, a.bias_entries);
        logits_each<THREADS>(a.bias_tokens, named.begin, named.end, [&](uint64_t i, int64_t token) {
            const uint64_t slot = static_cast<uint64_t>(token) - first;
            if (token >= 0 && slot < wide)
                atomicMax(&entries[slot], static_cast<uint32_t>(i - named.begin) + 1);
        });
    }
    __syncthreads();
    const float repetition = a.repetition ? a.repetition[row] : 1.0f;
    const float frequency = a.frequency ? a.frequency[row] : 0.0f;
    const float presence = a.presence ? a.presence[row] : 0.0f;
    const int32_t *mask = nullptr;
    if (a.masks) {
        const int32_t id = a.mask_ids[row];
        if (id >= 0 && static_cast<uint32_t>(id) < a.mask_count)
            mask = a.masks + static_cast<uint64_t>(id) * a.mask_words;
    }
#pragma unroll
    for (uint32_t quad = 0; quad < kQuads; ++quad) {
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {
            const uint32_t i = place(quad, c);
            if (i >= wide)
                continue;
            float &v = x[quad][c];
            const uint32_t count = counts[i], entry = entries[i];
            if (count) {
                v = v > 0.0f ? v / repetition : v * repetition;
                v = v - frequency * static_cast<float>(count);
                v = v - presence;
            }
            if (entry)
                v = v + a.bias_values[named.begin + entry - 1];
            if (mask) {
                const uint32_t token = first + i;
                if (!((static_cast<uint32_t>(mask[token >> 5]) >> (token & 31u)) & 1u))
                    v = -__builtin_inff();
            }
            if constexpr (!WIDE)
                a.out[at + i] = v;
        }
        if constexpr (WIDE)
            if (place(quad, 0) < wide)
                *reinterpret_cast<float4 *>(a.out + at + place(quad, 0)) = make_float4(x[quad][0], x[quad][1], x[quad][2], x[quad][3]);
    }
}

}  // namespace nz
