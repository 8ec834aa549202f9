// What the host sides of the C ABI share: errors, the layout of a blob, and where its sections are.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "neuzip.h"

#include "neuzip_format.h"

namespace nz {

extern thread_local int g_last_hip_error;  // of the last failing HIP call on this host thread

inline bool hip_ok(hipError_t e)
{
    if (e != hipSuccess) {
        g_last_hip_error = static_cast<int>(e);
        return false;
    }
    return true;
}
#define NZ_HIP(call)                 \
    do {                             \
        if (!hip_ok(call))           \
            return NEUZIP_EHIP;      \
    } while (0)

// A launch's threads in one dimension are fewer than 2^32.
constexpr bool too_many_wgs(uint64_t wgs, uint32_t threads) { return wgs >= (1ull << 32) / threads; }

constexpr uint64_t pad_to(uint64_t v, uint64_t a) { return (v + a - 1) / a * a; }
inline bool valid_k(int k) { return k == 7 || k == 3 || k == 1 || k == 0; }
inline uint64_t signmant_bytes(uint64_t n, int k) { return (n * static_cast<uint64_t>(k + 1) + 7) / 8; }
inline uint32_t chunks_of(uint64_t n) { return static_cast<uint32_t>((n + kChunk - 1) / kChunk); }

inline bool valid_block(uint32_t b) { return b == 32 || b == 64 || b == 128 || b == 256 || b == 512; }
inline uint64_t block_count(uint64_t n, uint32_t block) { return block ? (n + block - 1) / block : 0; }

struct Layout {
    uint64_t offsets, states, lens, mid_states, mid_lens, sm, low, coef, total;  // byte positions inside the fixed allocation
};

// f32: the tensor's elements are binary32; the plane of their lower halves follows the sign|mantissa stream
inline Layout fixed_layout(uint64_t n, int k, uint32_t block, bool f32)
{
    const uint64_t nc = chunks_of(n);
    Layout l;
    l.offsets = table_bytes(holds_table(chunks_of(n)));
    l.states = l.offsets + pad_to((nc + 2) * 4, 256);
    l.lens = l.states + pad_to(nc * kStates * 4, 256);
    const uint64_t entries = has_entry_points(chunks_of(n)) ? nc * kStates : 0;
    l.mid_states = l.lens + pad_to(nc * kStates, 256);
    l.mid_lens = l.mid_states + pad_to(entries * 4, 256);
    l.sm = l.mid_lens + pad_to(entries, 256);
    l.low = l.sm + pad_to(signmant_bytes(n, k), 256) + 256;
    l.coef = l.low + (f32 ? pad_to(n * 2, 256) + 256 : 0);
    l.total = l.coef + pad_to(block_count(n, block), 256);
    return l;
}

struct Container {
    uint64_t freq, offsets, states, lens, words, sm, low, coef, total;  // byte positions in the flat container
};

inline Container container_layout(uint64_t n, int k, uint64_t total_words, uint32_t block, bool f32)
{
    const uint64_t nc = chunks_of(n);
    Container c;
    c.freq = kHeaderBytes;
    c.offsets = c.freq + 512;
    c.states = c.offsets + pad_to((nc + 1) * 4, 16);
    c.lens = c.states + nc * kStates * 4;
    c.words = c.lens + nc * kStates;
    c.sm = c.words + pad_to(total_words * 2, 16);
    c.low = c.sm + pad_to(signmant_bytes(n, k), 16);
    c.coef = c.low + (f32 ? pad_to(n * 2, 16) : 0);
    c.total = c.coef + pad_to(block_count(n, block), 16);
    return c;
}

}  // namespace nz

struct neuzip_blob {
    uint32_t magic;
    int device;
    uint64_t n;
    int k;
    uint32_t block;  // block size of the block-wise normalisation, 0 = none
    uint32_t guard;  // guard band of the frequency table, 0 = none
    int elem;        // NEUZIP_BF16; NEUZIP_F32 (lossless only: a plane of lower halves rides along); NEUZIP_F16 (lossless only)
    bool has_table;  // holds a compressed tensor (and so a table that recompression can reuse)
    uint32_t n_chunks;
    uint64_t total_words;
    uint8_t *fixed;
    uint64_t fixed_bytes;
    uint8_t *words;
    uint64_t words_bytes;  // capacity of the word allocation
    uint64_t filled_by;    // number of the compress call that filled it, whose last kernels may still run ...
    hipStream_t filled_on; // ... on this stream (0 and nullptr: the host has waited for them)
    nz::Layout at;
    bool have_counts;
    uint32_t h_counts[256];
    uint16_t h_freq[256];
};

namespace nz {

constexpr uint32_t kBlobMagic = 0x424C5A4Eu;

inline TableBlock *table_of(const neuzip_blob *b) { return reinterpret_cast<TableBlock *>(b->fixed); }
inline uint32_t *offsets_of(const neuzip_blob *b) { return reinterpret_cast<uint32_t *>(b->fixed + b->at.offsets); }
inline uint32_t *states_of(const neuzip_blob *b) { return reinterpret_cast<uint32_t *>(b->fixed + b->at.states); }
inline uint8_t *lens_of(const neuzip_blob *b) { return b->fixed + b->at.lens; }
// (nullptr for blobs without entry points)
inline uint32_t *mid_states_of(const neuzip_blob *b)
{
    return has_entry_points(b->n_chunks) ? reinterpret_cast<uint32_t *>(b->fixed + b->at.mid_states) : nullptr;
}
inline uint8_t *mid_lens_of(const neuzip_blob *b)
{
    return has_entry_points(b->n_chunks) ? b->fixed + b->at.mid_lens : nullptr;
}
inline uint8_t *sm_of(const neuzip_blob *b) { return b->fixed + b->at.sm; }
inline uint8_t *coef_of(const neuzip_blob *b) { return b->fixed + b->at.coef; }
inline uint16_t *low_of(const neuzip_blob *b) { return reinterpret_cast<uint16_t *>(b->fixed + b->at.low); }
inline bool is_blob(const neuzip_blob *b) { return b && b->magic == kBlobMagic; }

// A blob lives on the device that was current when it was made; kernels are launched on the
// current device, so the two must agree.
inline bool on_current_device(const neuzip_blob *b)
{
    int cur = -1;
    return hipGetDevice(&cur) == hipSuccess && cur == b->device;
}

// Orders what `stream` is given next behind the calls that filled the blobs.  Calls that read a blob on the stream that it was
// filled on, or after the next compress call has reported, find nothing to do.  A stream under capture is left as it is.
int follow(const neuzip_blob *const *blobs, uint32_t count, hipStream_t stream);
inline int follow(const neuzip_blob *blob, hipStream_t stream) { return follow(&blob, 1, stream); }

// neuzip_linear_batch_scratch with another's work beside the layer's own.  launch, if there is one: launches the layer's kernel for the
// first tile of tokens (launch_linear), and whatever else can go beside it, on the stream.
struct LinearBatchArgs;
struct LinearLaunch;
typedef int (*LinearLauncher)(const LinearBatchArgs &batch, const LinearLaunch &kind, const void *context, hipStream_t stream);
int linear_with(const neuzip_blob *const *weights, const uint64_t *out_features, uint32_t count, uint64_t in_features,
                const void *d_x, uint32_t tokens, const float *const *d_bias, float *const *d_y, void *d_scratch,
                uint64_t scratch_bytes, LinearLauncher launch, const void *context, hipStream_t stream);

}  // namespace nz
