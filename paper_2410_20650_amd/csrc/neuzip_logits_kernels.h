// Penalties, biases and masks on logits for gfx950.
//
// One pass over the logits, a slice of a row's tokens to a workgroup.  The workgroup first counts, in LDS, how often each token of its slice
// occurs in the row's history, and finds the last bias entry of each; both with integer atomics, whose order does not show.  Every workgroup of a
// row reads the whole history (8 bytes a token, from the second one on out of a cache), which is why a slice is not shorter than it has to be for
// all CUs to have one.  What bounds it: reading and writing the logits once; for one row, the launch and the history's way through the caches.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace nz {

constexpr uint32_t kLogitsThreads = 256;

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

template <int SLICE>
__global__ void __launch_bounds__(kLogitsThreads) logits_kernel(const LogitsArgs a)
{
#pragma clang fp contract(off)
    __shared__ uint32_t counts[SLICE], entries[SLICE];  // entries: one more than the last entry's number in the row, 0: none
    const uint32_t row = blockIdx.y, first = blockIdx.x * SLICE;
    const uint32_t wide = a.vocab - first < SLICE ? a.vocab - first : SLICE;
    const bool counted = a.history != nullptr, biased = a.bias_tokens != nullptr;
    for (uint32_t i = threadIdx.x; i < SLICE; i += kLogitsThreads)
        counts[i] = entries[i] = 0;
    __syncthreads();
    LogitsRange named = {0, 0};
    if (counted) {
        const LogitsRange r = logits_range(a.history_starts, row, a.history_tokens);
        for (uint64_t i = r.begin + threadIdx.x; i < r.end; i += kLogitsThreads) {
            const uint64_t at = static_cast<uint64_t>(a.history[i]) - first;
            if (at < wide)
                atomicAdd(&counts[at], 1u);
        }
    }
    if (biased) {
        named = logits_range(a.bias_starts, row, a.bias_entries);
        for (uint64_t i = named.begin + threadIdx.x; i < named.end; i += kLogitsThreads) {
            const uint64_t at = static_cast<uint64_t>(a.bias_tokens[i]) - first;
            if (at < wide)
                atomicMax(&entries[at], static_cast<uint32_t>(i - named.begin) + 1);
        }
    }
    __syncthreads();
    const float repetition = a.repetition ? a.repetition[row] : 1.0f;
    const float frequency = a.frequency ? a.frequency[row] : 0.0f;
    const float presence = a.presence ? a.presence[row] : 0.0f;
    const int32_t *mask = nullptr;
    if (a.masks) {
        const int32_t id = a.mask_ids[row];
        if (id >= 0 && static_cast<uint32_t>(id) < a.mask_count)
            mask = a.masks + id * a.mask_words;
    }
    const uint64_t at = static_cast<uint64_t>(row) * a.vocab + first;
    for (uint32_t i = threadIdx.x; i < wide; i += kLogitsThreads) {
        float x = a.logits[at + i];
        const uint32_t count = counts[i], entry = entries[i];
        if (count) {
            x = x > 0.0f ? x / repetition : x * repetition;
            x = x - frequency * static_cast<float>(count);
            x = x - presence;
        }
        if (entry)
            x = x + a.bias_values[named.begin + entry - 1];
        if (mask) {
            const uint32_t token = first + i;
            if (!((static_cast<uint32_t>(mask[token >> 5]) >> (token & 31u)) & 1u))
                x = -__builtin_inff();
        }
        a.out[at + i] = x;
    }
}

}  // namespace nz
