// Cache of 8-bit keys and values, and the attention that reads it: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "neuzip.h"

#include "neuzip_attention_kernels.h"
#include "neuzip_attention_shape.h"
#include "neuzip_cache_kernels.h"
#include "neuzip_host.h"

using namespace nz;

namespace {

constexpr uint64_t kAttendMostRows = 1ull << 27;  // rows times query heads
constexpr float kLog2e = 1.4426950408889634f;

inline bool off(const void *p, uintptr_t size) { return reinterpret_cast<uintptr_t>(p) & (size - 1); }

inline bool valid_cache(const neuzip_cache *c)
{
    return c && c->d_k && c->d_v && c->d_k_scales && c->d_v_scales && !off(c->d_k, 16) && !off(c->d_v, 16) && !off(c->d_k_scales, 4) &&
           !off(c->d_v_scales, 4) && c->pages > 0 && c->pages < (1u << 31) && c->heads > 0 && (c->head_dim == 64 || c->head_dim == 128) &&
           (c->page_tokens == 16 || c->page_tokens == 32 || c->page_tokens == 64 || c->page_tokens == 128);
}

inline uint32_t page_shift(const neuzip_cache *c) { return __builtin_ctz(c->page_tokens); }

// positions are 32-bit numbers
inline bool valid_sequences(const neuzip_cache *c, const neuzip_sequences *s)
{
    return s && s->count < (1u << 24) && (s->count == 0 || (s->d_starts && s->d_lengths && s->d_table && s->table_width > 0)) && !off(s->d_starts, 4) &&
           !off(s->d_lengths, 4) && !off(s->d_table, 4) && (static_cast<uint64_t>(s->table_width) << page_shift(c)) < (1ull << 31);
}

inline SequencesView view_of(const neuzip_cache *c, const neuzip_sequences *s, uint32_t rows)
{
    return {s->d_starts, s->d_lengths, s->d_table, s->count, s->table_width, rows, page_shift(c), c->pages};
}

inline CacheView view_of(const neuzip_cache *c)
{
    return {static_cast<uint8_t *>(c->d_k), static_cast<uint8_t *>(c->d_v), c->d_k_scales, c->d_v_scales, c->heads};
}

inline bool valid_rows(const void *p, uint64_t row, uint64_t least, uint32_t size) { return p && !off(p, 16) && row >= least && row * size % 16 == 0 && row < (1ull << 31); }

template <class T, uint32_t DIM>
void launch_append(const AppendArgs &a, uint32_t wgs, hipStream_t stream)
{
    const uint32_t values = DIM << a.s.page_shift;
    if (values <= 16 * kAppendThreads)
        hipLaunchKernelGGL((append_kernel<T, DIM, 1>), dim3(wgs), dim3(kAppendThreads), 0, stream, a);
    else if (values <= 2 * 16 * kAppendThreads)
        hipLaunchKernelGGL((append_kernel<T, DIM, 2>), dim3(wgs), dim3(kAppendThreads), 0, stream, a);
    else if constexpr (DIM > 64)  // (64 * 128 fit two)
        hipLaunchKernelGGL((append_kernel<T, DIM, 4>), dim3(wgs), dim3(kAppendThreads), 0, stream, a);
}

inline AttendShape shape_of(const neuzip_cache *c, const neuzip_sequences *s, uint32_t q_heads, uint32_t rows, uint32_t window, uint64_t longest)
{
    const uint64_t room = static_cast<uint64_t>(s->table_width) << page_shift(c);
    return attend_shape(c->heads, c->head_dim, c->page_tokens, s->count, q_heads, rows, window, longest && longest < room ? longest : room);
}

inline bool valid_heads(const neuzip_cache *c, uint32_t q_heads) { return q_heads > 0 && q_heads % c->heads == 0; }

template <uint32_t DIM, bool WIDE>
void launch_attend_as(const AttendArgs &a, const AttendShape &shape, uint32_t wgs, hipStream_t stream)
{
    if (shape.rows == kAttendHugeRows) {
        if constexpr (WIDE && DIM == 128)  // (the rule's only case)
            hipLaunchKernelGGL((attend_many_kernel<DIM, WIDE, 8>), dim3(wgs), dim3(512), 0, stream, a);
    } else if (shape.rows == kAttendManyRows)
        hipLaunchKernelGGL((attend_many_kernel<DIM, WIDE, 4>), dim3(wgs), dim3(kAttendThreads), 0, stream, a);
    else if (shape.rows == kAttendSomeRows)
        hipLaunchKernelGGL((attend_some_kernel<DIM, WIDE>), dim3(wgs), dim3(kAttendThreads), 0, stream, a);
    else if (shape.waves == 8)
        hipLaunchKernelGGL((attend_few_kernel<DIM, 8, WIDE>), dim3(wgs), dim3(512), 0, stream, a);
    else
        hipLaunchKernelGGL((attend_few_kernel<DIM, 4, WIDE>), dim3(wgs), dim3(256), 0, stream, a);
}

template <uint32_t DIM>
int launch_attend(const AttendArgs &a, const AttendShape &shape, uint32_t wgs, hipStream_t stream)
{
    if ((1u << a.s.page_shift) >= kAttendStep)
        launch_attend_as<DIM, true>(a, shape, wgs, stream);
    else
        launch_attend_as<DIM, false>(a, shape, wgs, stream);
    if (!hip_ok(hipGetLastError()))
        return NEUZIP_EHIP;
    if (a.splits > 1) {
        constexpr uint32_t kAll = kAttendThreads / (DIM / 4);  // rows of a workgroup, or groups of a row
        const uint64_t count = static_cast<uint64_t>(a.s.rows) * a.q_heads;
        if (a.splits <= kAll)
            hipLaunchKernelGGL((attend_join_kernel<DIM, 1>), dim3(static_cast<uint32_t>((count + kAll - 1) / kAll)), dim3(kAttendThreads), 0, stream, a);
        else
            hipLaunchKernelGGL((attend_join_kernel<DIM, kAll>), dim3(static_cast<uint32_t>(count)), dim3(kAttendThreads), 0, stream, a);
        if (!hip_ok(hipGetLastError()))
            return NEUZIP_EHIP;
    }
    return NEUZIP_OK;
}

}  // namespace

extern "C" {

int neuzip_cache_append(const neuzip_cache *cache, const neuzip_sequences *sequences, int type, const void *d_k, uint64_t k_row,
                        const void *d_v, uint64_t v_row, const void *d_q, uint64_t q_row, uint32_t q_heads, void *d_q_out,
                        const float *d_rotary, uint64_t rotary_rows, uint32_t rows, void *hip_stream)
{
    if (!valid_cache(cache) || !valid_sequences(cache, sequences) || (type != NEUZIP_F32 && type != NEUZIP_BF16) || !d_q != !d_q_out ||
        rows >= (1u << 31))
        return NEUZIP_EINVAL;
    if (d_rotary && (off(d_rotary, 16) || rotary_rows < static_cast<uint64_t>(sequences->table_width) << page_shift(cache)))
        return NEUZIP_EINVAL;
    if (rows == 0 || sequences->count == 0)
        return NEUZIP_OK;
    const uint32_t size = type == NEUZIP_F32 ? 4 : 2;
    const uint64_t wide = static_cast<uint64_t>(cache->heads) * cache->head_dim;
    if (!valid_rows(d_k, k_row, wide, size) || !valid_rows(d_v, v_row, wide, size))
        return NEUZIP_EINVAL;
    if (d_q && (q_heads == 0 || !valid_rows(d_q, q_row, static_cast<uint64_t>(q_heads) * cache->head_dim, size) || off(d_q_out, 16)))
        return NEUZIP_EINVAL;
    const TileNumbers numbers = {page_shift(cache), 1, 2};
    const uint64_t tiles = tile_count(numbers, rows, sequences->count);
    const uint64_t wgs = tiles * cache->heads * 2 + (d_q ? rows : 0);
    if (cache->heads >= (1u << 16) || too_many_wgs(wgs, kAppendThreads))
        return NEUZIP_EUNSUPPORTED;
    AppendArgs a;
    a.s = view_of(cache, sequences, rows);
    a.c = view_of(cache);
    a.k = d_k;
    a.v = d_v;
    a.q = d_q;
    a.k_row = k_row;
    a.v_row = v_row;
    a.q_row = q_row;
    a.q_out = static_cast<uint16_t *>(d_q_out);
    a.rotary = d_rotary;
    a.q_heads = q_heads;
    a.tiles = static_cast<uint32_t>(tiles);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const uint32_t grid = static_cast<uint32_t>(wgs);
    if (type == NEUZIP_F32) {
        if (cache->head_dim == 64)
            launch_append<float, 64>(a, grid, stream);
        else
            launch_append<float, 128>(a, grid, stream);
    } else {
        if (cache->head_dim == 64)
            launch_append<uint16_t, 64>(a, grid, stream);
        else
            launch_append<uint16_t, 128>(a, grid, stream);
    }
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

uint64_t neuzip_cache_attention_scratch_bytes(const neuzip_cache *cache, const neuzip_sequences *sequences, uint32_t q_heads, uint32_t rows,
                                              uint32_t window, uint64_t longest)
{
    if (!valid_cache(cache) || !valid_sequences(cache, sequences) || !valid_heads(cache, q_heads) || rows == 0 || sequences->count == 0 ||
        static_cast<uint64_t>(rows) * q_heads >= kAttendMostRows)
        return 0;
    return shape_of(cache, sequences, q_heads, rows, window, longest).bytes;
}

int neuzip_cache_attention(const neuzip_cache *cache, const neuzip_sequences *sequences, const void *d_q, uint64_t q_row, uint32_t q_heads,
                           uint32_t rows, float scale, uint32_t window, uint64_t longest, void *d_out, void *d_scratch,
                           uint64_t scratch_bytes, void *hip_stream)
{
    if (!valid_cache(cache) || !valid_sequences(cache, sequences) || !valid_heads(cache, q_heads) || !(scale > 0.0f) || !std::isfinite(scale * kLog2e))
        return NEUZIP_EINVAL;
    if (rows == 0 || sequences->count == 0)
        return NEUZIP_OK;
    if (!valid_rows(d_q, q_row, static_cast<uint64_t>(q_heads) * cache->head_dim, 2) || !d_out || off(d_out, 16) || off(d_scratch, 16))
        return NEUZIP_EINVAL;
    if (static_cast<uint64_t>(rows) * q_heads >= kAttendMostRows)
        return NEUZIP_EUNSUPPORTED;
    const AttendShape shape = shape_of(cache, sequences, q_heads, rows, window, longest);
    if (shape.bytes && (!d_scratch || scratch_bytes < shape.bytes))
        return NEUZIP_EINVAL;
    const uint64_t wgs = shape.tiles * cache->heads * shape.splits;
    if (too_many_wgs(wgs, 512))
        return NEUZIP_EUNSUPPORTED;
    AttendArgs a;
    a.s = view_of(cache, sequences, rows);
    a.c = view_of(cache);
    a.q = static_cast<const uint16_t *>(d_q);
    a.q_row = q_row;
    a.out = static_cast<uint16_t *>(d_out);
    a.partial = static_cast<float *>(d_scratch);
    a.stats = reinterpret_cast<float2 *>(static_cast<uint8_t *>(d_scratch) + shape.sums);
    a.q_heads = q_heads;
    a.group = q_heads / cache->heads;
    a.window = window;
    a.splits = shape.splits;
    a.tiles = static_cast<uint32_t>(shape.tiles);
    a.numbers = shape.numbers;
    a.most_keys = shape.keys;
    a.least_steps = shape.least_steps;
    a.scale = scale * kLog2e;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const uint32_t grid = static_cast<uint32_t>(wgs);
    return cache->head_dim == 64 ? launch_attend<64>(a, shape, grid, stream) : launch_attend<128>(a, shape, grid, stream);
}

}  // extern "C"
