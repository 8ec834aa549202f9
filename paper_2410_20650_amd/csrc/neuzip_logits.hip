// Penalties, biases and masks on logits: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cstdint>

#include "neuzip.h"

#include "neuzip_host.h"
#include "neuzip_logits_kernels.h"

using namespace nz;

namespace {

constexpr uint32_t kLogitsMostRows = 65535;  // a grid's second dimension
// From so many logits on there is a long slice for each CU; a long one reads the row's history once for four times as many tokens.  us, rows of 128256 tokens with
// 2000 of history, short / long: 1 row 3.3 / 3.9, 8 rows 4.3 / 4.4, 12 rows 5.5 / 5.0, 48 rows 13.8 / 12.4.
constexpr uint64_t kLogitsMany = 256 * 4096;
constexpr uint64_t kLogitsMostEntries = 0xFFFFFFFEull;

inline bool off(const void *p, uintptr_t size) { return reinterpret_cast<uintptr_t>(p) & (size - 1); }

template <uint32_t SLICE, uint32_t THREADS>
void launch_logits(const LogitsArgs &a, uint32_t rows, bool wide, hipStream_t stream)
{
    const dim3 wgs((a.vocab + SLICE - 1) / SLICE, rows);
    if (wide)
        hipLaunchKernelGGL((logits_kernel<SLICE, THREADS, true>), wgs, dim3(THREADS), 0, stream, a);
    else
        hipLaunchKernelGGL((logits_kernel<SLICE, THREADS, false>), wgs, dim3(THREADS), 0, stream, a);
}

}  // namespace

extern "C" {

int neuzip_logits(const float *d_logits, uint32_t rows, uint64_t vocab, const int64_t *d_history, uint64_t history_tokens,
                  const int32_t *d_history_starts, const float *d_repetition, const float *d_frequency, const float *d_presence,
                  const int64_t *d_bias_tokens, const float *d_bias_values, uint64_t bias_entries, const int32_t *d_bias_starts,
                  const int32_t *d_masks, uint32_t masks, const int32_t *d_mask_ids, float *d_out, void *hip_stream)
{
    if (vocab == 0 || !d_masks != !d_mask_ids || (d_masks && masks == 0) || masks >= (1u << 31))
        return NEUZIP_EINVAL;
    // (a history or a list of biases without entries need not have memory)
    if (history_tokens && (!d_history || !d_history_starts))
        return NEUZIP_EINVAL;
    if (bias_entries && (!d_bias_tokens || !d_bias_values || !d_bias_starts))
        return NEUZIP_EINVAL;
    if (rows == 0)
        return NEUZIP_OK;
    if (!d_logits || !d_out)
        return NEUZIP_EINVAL;
    const void *const words[] = {d_logits, d_history_starts, d_repetition, d_frequency, d_presence, d_bias_values, d_bias_starts, d_masks, d_mask_ids, d_out};
    for (const void *p : words)
        if (off(p, 4))
            return NEUZIP_EINVAL;
    if (off(d_history, 8) || off(d_bias_tokens, 8))
        return NEUZIP_EINVAL;
    if (vocab >= (1ull << 31) || rows > kLogitsMostRows || bias_entries > kLogitsMostEntries)
        return NEUZIP_EUNSUPPORTED;
    LogitsArgs a;
    a.logits = d_logits;
    a.out = d_out;
    a.history = history_tokens ? d_history : nullptr;
    a.history_starts = d_history_starts;
    a.repetition = d_repetition;
    a.frequency = d_frequency;
    a.presence = d_presence;
    a.bias_tokens = bias_entries ? d_bias_tokens : nullptr;
    a.bias_values = d_bias_values;
    a.bias_starts = d_bias_starts;
    a.masks = d_masks;
    a.mask_ids = d_mask_ids;
    a.history_tokens = history_tokens;
    a.bias_entries = bias_entries;
    a.mask_words = (vocab + 31) / 32;
    a.mask_count = masks;
    a.vocab = static_cast<uint32_t>(vocab);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool wide = vocab % 4 == 0 && !off(d_logits, 16) && !off(d_out, 16);
    if (static_cast<uint64_t>(rows) * vocab >= kLogitsMany)
        launch_logits<4096, 512>(a, rows, wide, stream);
    else
        launch_logits<1024, 256>(a, rows, wide, stream);
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

}  // extern "C"
