// Attention over a cache of 8-bit keys and values for gfx950:  out = softmax(scale q K^T + mask) V  in one pass over the keys, with the running
// maximum and sum of each row.
//
// The query heads that read one head of the cache, and a sequence's newest tokens, are the rows of one product:  row r is token r / group, head
// r % group.  Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane of the matrix cores' results holds keys of one row:
// the weights P^T are then, once rounded to bf16, the second product's operand where they are, without a way through LDS.  For that the keys
// are taken in an order of their own (the sum over them has none): lane group g of four has keys 16 g .. 16 g + 15 of the 64 of a step,
// which in a page of the values are 16 consecutive bytes.  Bytes become bf16, times their page's scale, by one instruction for two (exact: e4m3 has 4
// significant bits and scales are powers of two).
//
// attend_few_kernel: a workgroup has up to 16 rows, a wave every fourth step of 64 keys, keys and values from memory straight into registers; the four
// waves' sums are joined in LDS.  Work is split over the keys too where there are few rows, and joined by attend_join_kernel.
// What bounds it: the bytes of the cache.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "neuzip_cache_kernels.h"

namespace nz {

constexpr uint32_t kAttendThreads = 256;
constexpr uint32_t kAttendFewRows = 16;
constexpr uint32_t kAttendStep = 64;      // keys
constexpr uint32_t kAttendLeastSteps = 4; // of a split: one for each wave

struct AttendArgs {
    SequencesView s;
    CacheView c;
    const uint16_t *q;
    uint64_t q_row;
    uint16_t *out;
    float *partial;     // splits > 1: sums of one split after the other, row by row, head_dim floats each ...
    float2 *stats;      // ... and the rows' maximum and sum
    uint32_t q_heads, group;
    uint32_t window;
    uint32_t splits;
    float scale;        // times log2(e)
};

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 attend_bf16x8_t;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 attend_bf16x2_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float attend_f32x4_t;

__device__ __forceinline__ float attend_exp2(float v) { return __builtin_amdgcn_exp2f(v); }

// eight bytes, times scale
__device__ __forceinline__ attend_bf16x8_t attend_widen(uint32_t a, uint32_t b, float scale)
{
    const attend_bf16x2_t w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false), x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
    const attend_bf16x2_t y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false), z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
    return attend_bf16x8_t{w[0], w[1], x[0], x[1], y[0], y[1], z[0], z[1]};
}

__device__ __forceinline__ attend_bf16x8_t attend_round(float a, float b, float c, float d, float e, float f, float g, float h)
{
    typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8_t;
    return __builtin_convertvector((f32x8_t{a, b, c, d, e, f, g, h}), attend_bf16x8_t);
}

// the bytes begin .. end - 1 of 16, byte 4 * word on
__device__ __forceinline__ uint32_t attend_bytes(int32_t begin, int32_t end, int32_t word)
{
    const int32_t a = begin - 4 * word, b = end - 4 * word;
    const uint32_t from = a <= 0 ? 0xFFFFFFFFu : a >= 4 ? 0u : 0xFFFFFFFFu << 8 * a;
    const uint32_t upto = b >= 4 ? 0xFFFFFFFFu : b <= 0 ? 0u : ~(0xFFFFFFFFu << 8 * b);
    return from & upto;
}

// bit 7 of the bytes that are NaN
__device__ __forceinline__ uint32_t attend_nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

// Which keys the rows of a tile see.
struct AttendRange {
    uint32_t low, high;          // any row: low .. high - 1
    uint32_t low_all, high_all;  // every row: low_all .. high_all - 1
};
// rows first_row .. last_row of a sequence
__device__ __forceinline__ AttendRange attend_range(const NewTokens &n, uint32_t first_token, uint32_t last_token, uint32_t window)
{
    const uint32_t first = n.first + first_token + 1, last = n.first + last_token + 1;  // one behind the last key
    AttendRange r;
    r.high = last;
    r.high_all = first;
    r.low = window && first > window ? first - window : 0;
    r.low_all = window && last > window ? last - window : 0;
    if (n.length == 0)
        r.low = r.high = r.low_all = r.high_all = 0;
    return r;
}

// The steps begin .. end - 1 of split `split` of the steps that the keys of r take.
__device__ __forceinline__ void attend_split(const AttendRange &r, uint32_t split, uint32_t splits, uint32_t &begin, uint32_t &end)
{
    const uint32_t first = r.low / kAttendStep, last = (r.high + kAttendStep - 1) / kAttendStep;
    uint32_t each = (last - first + splits - 1) / splits;
    each = each > kAttendLeastSteps ? each : kAttendLeastSteps;
    begin = first + split * each;
    begin = begin < last ? begin : last;
    end = last - begin > each ? begin + each : last;
}

// Where the sums of a row go: index of its token's head.
__device__ __forceinline__ uint64_t attend_row(const AttendArgs &a, const NewTokens &n, uint32_t head, uint32_t r)
{
    return static_cast<uint64_t>(n.begin + r / a.group) * a.q_heads + head * a.group + r % a.group;
}

template <uint32_t DIM>
__global__ void __launch_bounds__(kAttendThreads) attend_few_kernel(const AttendArgs a)
{
    constexpr uint32_t kWide = DIM / 64, kFeatures = DIM / 16, kWaves = kAttendThreads / 64, kStride = DIM + 4;
    __shared__ float sums[kWaves][kAttendFewRows][kStride];
    __shared__ float2 stats[kWaves][kAttendFewRows];
    const uint32_t split = blockIdx.x % a.splits, head = blockIdx.x / a.splits % a.c.heads, tile = blockIdx.x / a.splits / a.c.heads;
    const TileNumbers numbers = {kAttendFewRows, a.group, 1};
    const uint32_t s = sequence_of(a.s.starts, a.s.count, numbers, tile);
    if (s >= a.s.count)
        return;
    const NewTokens n = new_tokens(a.s, s);
    const uint64_t row0_wide = (tile - first_tile(numbers, a.s.starts[s], s)) * kAttendFewRows;
    const uint32_t rows = n.count * a.group;
    if (row0_wide >= rows)
        return;
    const uint32_t row0 = static_cast<uint32_t>(row0_wide), row_end = rows - row0 < kAttendFewRows ? rows : row0 + kAttendFewRows;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, i = lane % 16, g = lane / 16;
    const AttendRange range = attend_range(n, row0 / a.group, (row_end - 1) / a.group, a.window);

    // the lane's row: its query, and the keys that it sees
    const bool mine = row0 + i < row_end;
    const uint32_t row = mine ? row0 + i : row0, position = n.first + row / a.group;
    const uint32_t my_high = mine ? position + 1 : 0, my_low = a.window && position + 1 > a.window ? position + 1 - a.window : 0;
    attend_bf16x8_t q[kWide][2];
    const uint16_t *q_at = a.q + (n.begin + row / a.group) * a.q_row + (head * a.group + row % a.group) * DIM + g * 16;
#pragma unroll
    for (uint32_t j = 0; j < kWide; ++j)
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h)
            q[j][h] = *reinterpret_cast<const attend_bf16x8_t *>(q_at + j * 64 + h * 8);

    attend_f32x4_t o[kFeatures] = {};
    float top = -__builtin_inff(), total = 0.0f;
    uint32_t step, last;
    attend_split(range, split, a.splits, step, last);
    const uint32_t shift = a.s.page_shift, inside = (1u << shift) - 1;
    for (step += wave; step < last; step += kWaves) {
        const uint32_t k0 = step * kAttendStep;
        const uint32_t k_group = k0 + i / 4 * 16, v_group = k0 + g * 16;
        const bool k_there = k_group < range.high && k_group + 16 > range.low, v_there = v_group < range.high && v_group + 16 > range.low;
        uint32_t k_page = k_there ? page_of(a.s, s, k_group >> shift) : kNoPage, v_page = v_there ? page_of(a.s, s, v_group >> shift) : kNoPage;
        const bool held = v_page != kNoPage;
        k_page = k_page != kNoPage ? k_page : 0;  // (read, and not used)
        v_page = held ? v_page : 0;
        const uint64_t k_head = static_cast<uint64_t>(k_page) * a.c.heads + head, v_head = static_cast<uint64_t>(v_page) * a.c.heads + head;
        const uint8_t *k_at = a.c.k + ((k_head << shift) + (k_group & inside) + i % 4) * DIM + g * 16;
        const uint8_t *v_at = a.c.v + ((v_head * DIM + i) << shift) + (v_group & inside);
        const float k_scale = a.c.k_scales[k_head], v_scale = held ? a.c.v_scales[v_head] : 1.0f;
        uint4 k[4][kWide], v[kFeatures];
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t j = 0; j < kWide; ++j)
                k[t][j] = *reinterpret_cast<const uint4 *>(k_at + t * 4 * DIM + j * 64);
#pragma unroll
        for (uint32_t f = 0; f < kFeatures; ++f)
            v[f] = *reinterpret_cast<const uint4 *>(v_at + (static_cast<uint64_t>(f) * 16 << shift));
        attend_f32x4_t score[4] = {};
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t j = 0; j < kWide; ++j) {
                score[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(k[t][j].x, k[t][j].y, k_scale), q[j][0], score[t], 0, 0, 0);
                score[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(k[t][j].z, k[t][j].w, k_scale), q[j][1], score[t], 0, 0, 0);
            }
        // at an edge: what a row does not see, and values that no row sees (whatever is there may be NaN, and 0 * NaN is)
        const bool edge = k0 < range.low_all || k0 + kAttendStep > range.high_all || __any(!held);
        uint32_t nans = 0;
        if (edge) {
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r) {
                    const uint32_t key = v_group + t * 4 + r;
                    if (!(held && key >= my_low && key < my_high))
                        score[t][r] = -__builtin_inff();
                }
            const int32_t from = held ? static_cast<int32_t>(range.low - v_group) : 16, upto = held ? static_cast<int32_t>(range.high - v_group) : 0;
            const uint32_t m0 = attend_bytes(from, upto, 0), m1 = attend_bytes(from, upto, 1), m2 = attend_bytes(from, upto, 2), m3 = attend_bytes(from, upto, 3);
#pragma unroll
            for (uint32_t f = 0; f < kFeatures; ++f) {
                v[f].x &= m0, v[f].y &= m1, v[f].z &= m2, v[f].w &= m3;
                nans |= attend_nan_bytes(v[f].x) | attend_nan_bytes(v[f].y) | attend_nan_bytes(v[f].z) | attend_nan_bytes(v[f].w);
            }
        }
        float most = -__builtin_inff();
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
                most = fmaxf(most, score[t][r]);
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float now = fmaxf(top, most * a.scale), base = now == -__builtin_inff() ? 0.0f : now;
        const float less = attend_exp2(top - base);
        top = now;
        total *= less;
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                score[t][r] = attend_exp2(score[t][r] * a.scale - base);
                total += score[t][r];
            }
#pragma unroll
        for (uint32_t f = 0; f < kFeatures; ++f)
            o[f] *= less;
        if (__any(nans != 0)) {
            // NaN among values that some rows see and others do not: the rows that see it have it
#pragma unroll
            for (uint32_t f = 0; f < kFeatures; ++f) {
                attend_f32x4_t seen = {};
                uint32_t w[4] = {v[f].x, v[f].y, v[f].z, v[f].w};
#pragma unroll
                for (uint32_t u = 0; u < 2; ++u) {
                    uint32_t is[2];
                    attend_bf16x8_t sees;
#pragma unroll
                    for (uint32_t b = 0; b < 2; ++b) {
                        const uint32_t bits = attend_nan_bytes(w[2 * u + b]);
                        is[b] = (bits >> 7) * 0x38u;  // 1.0
                        w[2 * u + b] &= ~((bits >> 7) * 0xFFu);
                    }
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e) {
                        const uint32_t key = v_group + u * 8 + e;
                        sees[e] = key >= my_low && key < my_high ? static_cast<__bf16>(1.0f) : static_cast<__bf16>(0.0f);
                    }
                    seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(is[0], is[1], 1.0f), sees, seen, 0, 0, 0);
                }
                v[f] = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
                for (uint32_t r = 0; r < 4; ++r)
                    o[f][r] = seen[r] > 0.0f ? __builtin_nanf("") : o[f][r];
            }
        }
        const attend_bf16x8_t p0 = attend_round(score[0][0], score[0][1], score[0][2], score[0][3], score[1][0], score[1][1], score[1][2], score[1][3]);
        const attend_bf16x8_t p1 = attend_round(score[2][0], score[2][1], score[2][2], score[2][3], score[3][0], score[3][1], score[3][2], score[3][3]);
#pragma unroll
        for (uint32_t f = 0; f < kFeatures; ++f) {
            o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(v[f].x, v[f].y, v_scale), p0, o[f], 0, 0, 0);
            o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(v[f].z, v[f].w, v_scale), p1, o[f], 0, 0, 0);
        }
    }
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    if (g == 0)
        stats[wave][i] = make_float2(top, total);
#pragma unroll
    for (uint32_t f = 0; f < kFeatures; ++f)
        *reinterpret_cast<attend_f32x4_t *>(&sums[wave][i][f * 16 + g * 4]) = o[f];
    __syncthreads();
    // sixteen lanes to a row
    const uint32_t r = threadIdx.x / 16, at = threadIdx.x % 16 * (DIM / 16);
    if (row0 + r >= row_end)
        return;
    float all = -__builtin_inff(), whole = 0.0f, sum[DIM / 16] = {};
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w)
        all = fmaxf(all, stats[w][r].x);
    const float base = all == -__builtin_inff() ? 0.0f : all;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        const float part = attend_exp2(stats[w][r].x - base);
        whole += part * stats[w][r].y;
#pragma unroll
        for (uint32_t d = 0; d < DIM / 16; ++d)
            sum[d] += part * sums[w][r][at + d];
    }
    const uint64_t to = attend_row(a, n, head, row0 + r);
    if (a.splits > 1) {
        const uint64_t place = static_cast<uint64_t>(split) * a.s.rows * a.q_heads + to;
        if (at == 0)
            a.stats[place] = make_float2(all, whole);
#pragma unroll
        for (uint32_t d = 0; d < DIM / 16; d += 4)
            *reinterpret_cast<float4 *>(a.partial + place * DIM + at + d) = make_float4(sum[d], sum[d + 1], sum[d + 2], sum[d + 3]);
        return;
    }
    const float once = whole == 0.0f ? 0.0f : 1.0f / whole;
#pragma unroll
    for (uint32_t d = 0; d < DIM / 16; d += 4) {
        typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
        const attend_f32x4_t v = {sum[d] * once, sum[d + 1] * once, sum[d + 2] * once, sum[d + 3] * once};
        *reinterpret_cast<bf16x4_t *>(a.out + to * DIM + at + d) = __builtin_convertvector(v, bf16x4_t);
    }
}

// The splits of a row together; four features to a lane.
template <uint32_t DIM>
__global__ void __launch_bounds__(kAttendThreads) attend_join_kernel(const AttendArgs a)
{
    constexpr uint32_t kLanes = DIM / 4, kRows = kAttendThreads / kLanes;
    const uint64_t count = static_cast<uint64_t>(a.s.rows) * a.q_heads;
    const uint64_t row = static_cast<uint64_t>(blockIdx.x) * kRows + threadIdx.x / kLanes;
    const uint32_t at = threadIdx.x % kLanes * 4;
    const int64_t token = static_cast<int64_t>(row / a.q_heads);
    if (row >= count || token < a.s.starts[0] || token >= a.s.starts[a.s.count])
        return;  // (a row of nobody's)
    float all = -__builtin_inff();
    for (uint32_t p = 0; p < a.splits; ++p)
        all = fmaxf(all, a.stats[p * count + row].x);
    const float base = all == -__builtin_inff() ? 0.0f : all;
    float whole = 0.0f;
    attend_f32x4_t sum = {};
    for (uint32_t p = 0; p < a.splits; ++p) {
        const float2 part = a.stats[p * count + row];
        const float share = attend_exp2(part.x - base);
        whole += share * part.y;
        sum += share * *reinterpret_cast<const attend_f32x4_t *>(a.partial + (p * count + row) * DIM + at);
    }
    typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
    sum *= whole == 0.0f ? 0.0f : 1.0f / whole;
    *reinterpret_cast<bf16x4_t *>(a.out + row * DIM + at) = __builtin_convertvector(sum, bf16x4_t);
}

}  // namespace nz
