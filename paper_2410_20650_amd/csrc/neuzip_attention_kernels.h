// Attention over a cache of 8-bit keys and values for gfx950:  out = softmax(scale q K^T + mask) V  in one pass over the keys, with the running
// maximum and sum of each row.
//
// The query heads that read one head of the cache, and a sequence's newest tokens, are the rows of one product:  row r is token r / group, head
// r % group.  Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane of the matrix cores' results holds keys of one row:
// the weights P^T are then, once rounded to bf16, the second product's operand where they are, without a way through LDS.  For that the keys
// are taken in an order of their own (the sum over them has none): lane group g of four has keys 16 g .. 16 g + 15 of the 64 of a step,
// which in a page of the values are 16 consecutive bytes.  Bytes become bf16, times their page's scale, by one instruction for two (exact: e4m3 has 4
// significant bits and scales are powers of two).  The weights are rounded because the matrix cores multiply bf16 by bf16; their sum is that of the unrounded ones, in
// binary32.  Against 64 bits the results are off by 0.0020 to 0.0023 of themselves (root mean square), where weights in binary32 have 0.0016 to 0.0017, what the
// rounding of the result takes alone.
//
// attend_few_kernel: a workgroup has up to 16 rows, its waves a step of 64 keys each in turn, keys and values from memory straight into registers; the
// waves' sums are joined in LDS.  Work is split over the keys too where there are few rows, and joined by attend_join_kernel.
// What bounds it: the bytes of the cache.  Measured, 32 query heads on 8 of 128: 32 sequences of 8192 tokens 93 us a call (5.8 TB/s), 48 of 2178 to 8192 108 (4.8: the
// longest ones' workgroups end last), one of 32768 tokens 14.3 us and 4.6 for the join of its 32 splits.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "neuzip_attention_shape.h"
#include "neuzip_cache_kernels.h"

namespace nz {

constexpr uint32_t kAttendThreads = 256;
// A row's weights may exceed 1 by so much (a factor of 64) before its sums are scaled down to a new maximum.  Each row goes by its own keys: were it scaled whenever
// another one of its wave is, its last bits would hang on keys that it does not see.
constexpr float kAttendSlack = 6.0f;

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
    uint32_t splits, tiles;
    TileNumbers numbers;  // of the tiles
    uint32_t most_keys;   // that a tile's rows see, as the caller has it
    uint32_t least_steps; // of a split
    float scale;        // times log2(e)
};

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 attend_bf16x8_t;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 attend_bf16x2_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float attend_f32x4_t;

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float attend_f32x16_t;

__device__ __forceinline__ float attend_max_of_halves(float v)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const auto both = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    const uint32_t low = both[0], high = both[1];  // (a bit cast of both[1] itself is taken for both[0]'s)
    return fmaxf(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high));
}

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

constexpr uint32_t kE4m3One = 0x38u;
// bit 7 of the bytes that are NaN
__device__ __forceinline__ uint32_t attend_nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
// The bytes outside `keep`, and NaN, made 0; not 0 if there was NaN.
__device__ __forceinline__ uint32_t attend_clean(uint32_t &w, uint32_t keep)
{
    w &= keep;
    const uint32_t nans = attend_nan_bytes(w);
    w &= ~((nans >> 7) * 0xFFu);
    return nans;
}

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

// Whether some row does not see all keys of the step from k0 on.
__device__ __forceinline__ bool attend_edge(const AttendRange &r, uint32_t k0) { return k0 < r.low_all || k0 + kAttendStep > r.high_all; }

// The steps begin .. end - 1 of split `split` of the steps that the keys of r take.  A split has as many steps in every sequence, the longest's
// divided by the splits: workgroups of a ragged batch are then equally long, short sequences have fewer of them.
__device__ __forceinline__ void attend_split(const AttendArgs &a, uint32_t longest, const AttendRange &r, uint32_t split, uint32_t &begin, uint32_t &end)
{
    const uint32_t first = r.low / kAttendStep, last = (r.high + kAttendStep - 1) / kAttendStep;
    if (a.splits == 1) {
        begin = first;
        end = last;
        return;
    }
    const uint32_t keys = longest < a.most_keys ? longest : a.most_keys;
    // (one step more: a window need not begin with a step.  At least so many that the splits hold all there are.)
    uint32_t each = ((keys + kAttendStep - 1) / kAttendStep + 1 + a.splits - 1) / a.splits;
    const uint32_t least = (last - first + a.splits - 1) / a.splits;
    each = each > least ? each : least;
    each = each > a.least_steps ? each : a.least_steps;
    begin = first + split * each;
    begin = begin < last ? begin : last;
    end = last - begin > each ? begin + each : last;
}

// What the table says of a page, asked for a step before it is needed.  It is looked at only then: a check right behind the request would wait for it, and
// for the keys and values that were requested before it.
struct AttendEntry {
    uint32_t page;
    bool in;
};
// 0 that is a vector register: number + 0 for a vector load.  Scalar loads, the compiler's choice where all lanes ask for one number, are waited for together with
// all that comes from LDS; but the first answer of all is there sooner by one.
__device__ __forceinline__ uint32_t attend_zero()
{
    uint32_t zero;
    asm volatile("v_mov_b32 %0, 0" : "=v"(zero));
    return zero;
}
__device__ __forceinline__ AttendEntry attend_ask(const SequencesView &v, uint32_t s, uint32_t number, bool wanted, uint32_t zero = 0)
{
    AttendEntry e;
    e.in = wanted && number < v.table_width;
    e.page = static_cast<uint32_t>((v.table + static_cast<uint64_t>(s) * v.table_width + (e.in ? number : 0))[zero]);
    return e;
}
// UNIFORM: the number is the same for all lanes
template <bool UNIFORM>
__device__ __forceinline__ uint32_t attend_told(const SequencesView &v, const AttendEntry &e)
{
    const uint32_t page = UNIFORM ? __builtin_amdgcn_readfirstlane(e.page) : e.page;
    return e.in && page < v.pages ? page : kNoPage;
}

// Where the sums of a row go: index of its token's head.
__device__ __forceinline__ uint64_t attend_row(const AttendArgs &a, const NewTokens &n, uint32_t head, uint32_t r)
{
    return static_cast<uint64_t>(n.begin + r / a.group) * a.q_heads + head * a.group + r % a.group;
}

// The waves' sums of a workgroup's rows together, and out.
template <uint32_t DIM, uint32_t WAVES, uint32_t ROWS>
__device__ __forceinline__ void attend_leave(const AttendArgs &a, const NewTokens &n, uint32_t head, uint32_t split, uint32_t row0, uint32_t row_end,
                                             const float (&sums)[WAVES][ROWS][DIM + 4], const float2 (&stats)[WAVES][ROWS])
{
    // lanes that share a row, kOf features each
    constexpr uint32_t kOf = DIM * ROWS / (WAVES * 64);
    const uint32_t r = threadIdx.x / (DIM / kOf), at = threadIdx.x % (DIM / kOf) * kOf;
    if (row0 + r >= row_end)
        return;
    float all = -__builtin_inff(), whole = 0.0f, sum[kOf] = {};
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w)
        all = fmaxf(all, stats[w][r].x);
    const float base = all == -__builtin_inff() ? 0.0f : all;
#pragma unroll
    for (uint32_t w = 0; w < WAVES; ++w) {
        const float part = attend_exp2(stats[w][r].x - base);
        whole += part * stats[w][r].y;
#pragma unroll
        for (uint32_t d = 0; d < kOf; ++d)
            sum[d] += part * sums[w][r][at + d];
    }
    const uint64_t to = attend_row(a, n, head, row0 + r);
    if (a.splits > 1) {
        const uint64_t place = static_cast<uint64_t>(split) * a.s.rows * a.q_heads + to;
        if (at == 0)
            a.stats[place] = make_float2(all, whole);
#pragma unroll
        for (uint32_t d = 0; d < kOf; d += 2)
            *reinterpret_cast<float2 *>(a.partial + place * DIM + at + d) = make_float2(sum[d], sum[d + 1]);
        return;
    }
    const float once = whole == 0.0f ? 0.0f : 1.0f / whole;
#pragma unroll
    for (uint32_t d = 0; d < kOf; d += 2) {
        typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
        const f32x2_t v = {sum[d] * once, sum[d + 1] * once};
        *reinterpret_cast<attend_bf16x2_t *>(a.out + to * DIM + at + d) = __builtin_convertvector(v, attend_bf16x2_t);
    }
}

// Adds to `seen`, of every row, how many of the values of `feature` that it sees are NaN among 64 keys from k0 on (32 x 32 x 16).
__device__ __forceinline__ attend_f32x16_t attend_nans(const AttendArgs &a, uint32_t s, uint32_t head, uint32_t dim, uint32_t feature, uint32_t k0, uint32_t half,
                                                       uint32_t my_low, uint32_t my_high, attend_f32x16_t seen)
{
    const uint32_t shift = a.s.page_shift;
#pragma unroll 1
    for (uint32_t u = 0; u < 4; ++u) {
        const uint32_t key = k0 + u / 2 * 32 + half * 16 + u % 2 * 8, page = page_of(a.s, s, key >> shift);
        const uint64_t at = ((static_cast<uint64_t>(page != kNoPage ? page : 0) * a.c.heads + head) * dim + feature) << shift;
        const uint2 bytes = *reinterpret_cast<const uint2 *>(a.c.v + at + (key & ((1u << shift) - 1)));
        attend_bf16x8_t sees;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e)
            sees[e] = page != kNoPage && key + e >= my_low && key + e < my_high ? static_cast<__bf16>(1.0f) : static_cast<__bf16>(0.0f);
        const attend_bf16x8_t is = attend_widen((attend_nan_bytes(bytes.x) >> 7) * kE4m3One, (attend_nan_bytes(bytes.y) >> 7) * kE4m3One, 1.0f);
        seen = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is, sees, seen, 0, 0, 0);
    }
    return seen;
}

// WIDE: a step lies in one page
template <uint32_t DIM, uint32_t WAVES, bool WIDE>
__global__ void __launch_bounds__(WAVES * 64, 3) attend_few_kernel(const AttendArgs a)
{
    constexpr uint32_t kWide = DIM / 64, kFeatures = DIM / 16, kStride = DIM + 4;
    __shared__ float sums[WAVES][kAttendFewRows][kStride];
    __shared__ float2 stats[WAVES][kAttendFewRows];
    __shared__ attend_bf16x8_t queries[kWide * 2][64];
    const uint32_t split = blockIdx.x % a.splits, head = blockIdx.x / a.splits % a.c.heads, tile = blockIdx.x / a.splits / a.c.heads;
    const Found at = find_sequence(a.s, a.numbers, tile, a.splits > 1);
    if (at.s >= a.s.count)
        return;
    const uint32_t s = at.s;
    const NewTokens n = at.n;
    const uint64_t row0_wide = at.tile * kAttendFewRows;
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
    // (the query is read from LDS in every step: its 4 KB would be 16 registers of every wave, which three waves of a SIMD do not have)
    if (wave < kWide * 2) {
        const uint16_t *q_at = a.q + (n.begin + row / a.group) * a.q_row + (head * a.group + row % a.group) * DIM + g * 16;
        queries[wave][lane] = *reinterpret_cast<const attend_bf16x8_t *>(q_at + wave / 2 * 64 + wave % 2 * 8);
    }
    __syncthreads();

    attend_f32x4_t o[kFeatures] = {};
    float top = -__builtin_inff(), total = 0.0f;
    uint32_t step, last;
    attend_split(a, at.longest, range, split, step, last);
    // Requests run ahead of the sums: the next step's pages are looked up a step before, its keys are asked for as soon as this step's are
    // used up, its values behind this step's second product.
    const uint32_t shift = a.s.page_shift, inside = (1u << shift) - 1;
    AttendEntry k_entry, v_entry;
    const auto find_pages = [&](uint32_t at, uint32_t zero) {
        if constexpr (WIDE) {
            k_entry = v_entry = attend_ask(a.s, s, __builtin_amdgcn_readfirstlane(at * kAttendStep >> shift), at < last, zero);
            return;
        }
        const uint32_t k_group = at * kAttendStep + i / 4 * 16, v_group = at * kAttendStep + g * 16;
        k_entry = attend_ask(a.s, s, k_group >> shift, at < last && k_group < range.high && k_group + 16 > range.low);
        v_entry = attend_ask(a.s, s, v_group >> shift, at < last && v_group < range.high && v_group + 16 > range.low);
    };
    uint4 k[4][kWide], v[kFeatures];
    float k_scale, v_scale;
    bool held;
    uint32_t found = 0;  // NaN among values that not all rows see
    const auto request_keys = [&](uint32_t at) {
        const uint32_t k_page = attend_told<WIDE>(a.s, k_entry);
        const uint64_t page = static_cast<uint64_t>(k_page != kNoPage ? k_page : 0) * a.c.heads + head;  // (read, and not used)
        const uint8_t *from = WIDE ? a.c.k + ((page << shift) + (at * kAttendStep & inside)) * DIM + (i / 4 * 16 + i % 4) * DIM + g * 16
                                   : a.c.k + ((page << shift) + ((at * kAttendStep + i / 4 * 16) & inside) + i % 4) * DIM + g * 16;
        k_scale = a.c.k_scales[page];
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t j = 0; j < kWide; ++j)
                k[t][j] = *reinterpret_cast<const uint4 *>(from + t * 4 * DIM + j * 64);
    };
    // (and the entries of the step `next`, before the values: whoever waits for them does not wait for these)
    const auto request_values = [&](uint32_t at, uint32_t next) {
        const uint32_t v_page = attend_told<WIDE>(a.s, v_entry);
        held = v_page != kNoPage;
        find_pages(next, attend_zero());
        const uint64_t page = static_cast<uint64_t>(held ? v_page : 0) * a.c.heads + head;
        const uint8_t *from = WIDE ? a.c.v + (page * DIM << shift) + (at * kAttendStep & inside) + (i << shift) + g * 16
                                   : a.c.v + ((page * DIM + i) << shift) + ((at * kAttendStep + g * 16) & inside);
        v_scale = a.c.v_scales[page];
#pragma unroll
        for (uint32_t f = 0; f < kFeatures; ++f)
            v[f] = *reinterpret_cast<const uint4 *>(from + (f * 16 << shift));
    };
    step += wave;
    const uint32_t begin = step;
    if (step < last) {
        find_pages(step, 0);
        request_keys(step);
        request_values(step, step + WAVES);
    }
    for (; step < last; step += WAVES) {
        const uint32_t k0 = step * kAttendStep, v_group = k0 + g * 16;
        asm volatile("" ::: "memory");  // (it stays in LDS)
        attend_f32x4_t score[4] = {};
#pragma unroll
        for (uint32_t j = 0; j < kWide; ++j) {
            const attend_bf16x8_t first = queries[j * 2][lane], second = queries[j * 2 + 1][lane];
#pragma unroll
            for (uint32_t t = 0; t < 4; ++t) {
                score[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(k[t][j].x, k[t][j].y, k_scale), first, score[t], 0, 0, 0);
                score[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(k[t][j].z, k[t][j].w, k_scale), second, score[t], 0, 0, 0);
            }
        }
        // at an edge: what a row does not see; values that no row sees, and NaN (0 * NaN is), are made 0, and who sees NaN is looked up in the end
        if (step + WAVES < last)
            request_keys(step + WAVES);
        if (attend_edge(range, k0) || __any(!held)) {
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
            for (uint32_t f = 0; f < kFeatures; ++f)
                found |= attend_clean(v[f].x, m0) | attend_clean(v[f].y, m1) | attend_clean(v[f].z, m2) | attend_clean(v[f].w, m3);
        }
        float most = -__builtin_inff();
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
                most = fmaxf(most, score[t][r]);
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        most *= a.scale;
        if (__any(most > top + kAttendSlack)) {
            const float higher = most > top + kAttendSlack ? most : top, less = higher == -__builtin_inff() ? 1.0f : attend_exp2(top - higher);
            top = higher;
            total *= less;
#pragma unroll
            for (uint32_t f = 0; f < kFeatures; ++f)
                o[f] *= less;
        }
        const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
        for (uint32_t t = 0; t < 4; ++t)
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r) {
                score[t][r] = attend_exp2(score[t][r] * a.scale - base);
                total += score[t][r];
            }
        const attend_bf16x8_t p0 = attend_round(score[0][0], score[0][1], score[0][2], score[0][3], score[1][0], score[1][1], score[1][2], score[1][3]);
        const float of_values = held ? v_scale : 1.0f;
        const attend_bf16x8_t p1 = attend_round(score[2][0], score[2][1], score[2][2], score[2][3], score[3][0], score[3][1], score[3][2], score[3][3]);
#pragma unroll
        for (uint32_t f = 0; f < kFeatures; ++f) {
            o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(v[f].x, v[f].y, of_values), p0, o[f], 0, 0, 0);
            o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(attend_widen(v[f].z, v[f].w, of_values), p1, o[f], 0, 0, 0);
        }
        if (step + WAVES < last)
            request_values(step + WAVES, step + 2 * WAVES);
    }
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    if (__any(found != 0)) {
        // a row that sees a value that is NaN has it: products of where NaN is with who sees it
#pragma unroll
        for (uint32_t f = 0; f < kFeatures; ++f) {
            attend_f32x4_t seen = {};
            for (step = begin; step < last; step += WAVES)
#pragma unroll 1
                for (uint32_t u = 0; u < 2; ++u) {
                    const uint32_t key = step * kAttendStep + g * 16 + u * 8, page = page_of(a.s, s, key >> shift);
                    const uint64_t from = ((static_cast<uint64_t>(page != kNoPage ? page : 0) * a.c.heads + head) * DIM + f * 16 + i) << shift;
                    const uint2 bytes = *reinterpret_cast<const uint2 *>(a.c.v + from + (key & inside));
                    attend_bf16x8_t sees;
#pragma unroll
                    for (uint32_t e = 0; e < 8; ++e)
                        sees[e] = page != kNoPage && key + e >= my_low && key + e < my_high ? static_cast<__bf16>(1.0f) : static_cast<__bf16>(0.0f);
                    const attend_bf16x8_t is = attend_widen((attend_nan_bytes(bytes.x) >> 7) * kE4m3One, (attend_nan_bytes(bytes.y) >> 7) * kE4m3One, 1.0f);
                    seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(is, sees, seen, 0, 0, 0);
                }
#pragma unroll
            for (uint32_t r = 0; r < 4; ++r)
                o[f][r] = seen[r] > 0.0f ? __builtin_nanf("") : o[f][r];
        }
    }
    if (g == 0)
        stats[wave][i] = make_float2(top, total);
#pragma unroll
    for (uint32_t f = 0; f < kFeatures; ++f)
        *reinterpret_cast<attend_f32x4_t *>(&sums[wave][i][f * 16 + g * 4]) = o[f];
    __syncthreads();
    attend_leave<DIM, WAVES, kAttendFewRows>(a, n, head, split, row0, row_end, sums, stats);
}

// ---- some rows: the same with 32 rows to a workgroup, in matrix instructions of 32 x 32.  Here the lane (row c = l % 32, half h = l / 32) has of
// every 32 keys the ones 16 h .. 16 h + 15; row c of 32 of the keys' operand is key 16 * (c / 4 % 2) + 4 * (c / 8) + c % 4.  What bounds it: the way from a page's number
// to its bytes, a step or two after another for each wave.  Measured: 512 tokens, 32 query heads on 8 of 128, 11.6 us; 1405 of five sequences of 722 to 2011 tokens,
// 15 heads on 3 of 64, a window of 256, 12.1.

template <uint32_t DIM, bool WIDE>
__global__ void __launch_bounds__(kAttendThreads, 2) attend_some_kernel(const AttendArgs a)
{
    constexpr uint32_t kWide = DIM / 32, WAVES = kAttendThreads / 64, kStride = DIM + 4;
    __shared__ float sums[WAVES][kAttendSomeRows][kStride];
    __shared__ float2 stats[WAVES][kAttendSomeRows];
    __shared__ attend_bf16x8_t queries[kWide * 2][64];
    const uint32_t head = blockIdx.x % a.c.heads, split = blockIdx.x / a.c.heads % a.splits, tile = a.tiles - 1 - blockIdx.x / a.c.heads / a.splits;
    const Found at = find_sequence(a.s, a.numbers, tile, a.splits > 1);
    if (at.s >= a.s.count)
        return;
    const uint32_t s = at.s;
    const NewTokens n = at.n;
    const uint64_t row0_wide = at.tile * kAttendSomeRows;
    const uint32_t rows = n.count * a.group;
    if (row0_wide >= rows)
        return;
    const uint32_t row0 = static_cast<uint32_t>(row0_wide), row_end = rows - row0 < kAttendSomeRows ? rows : row0 + kAttendSomeRows;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, c = lane % 32, h = lane / 32;
    const AttendRange range = attend_range(n, row0 / a.group, (row_end - 1) / a.group, a.window);
    const bool mine = row0 + c < row_end;
    const uint32_t row = mine ? row0 + c : row0, position = n.first + row / a.group;
    const uint32_t my_high = mine ? position + 1 : 0, my_low = a.window && position + 1 > a.window ? position + 1 - a.window : 0;
    const uint16_t *q_at = a.q + (n.begin + row / a.group) * a.q_row + (head * a.group + row % a.group) * DIM + h * 16;
#pragma unroll
    for (uint32_t j = wave; j < kWide * 2; j += WAVES)
        queries[j][lane] = *reinterpret_cast<const attend_bf16x8_t *>(q_at + j / 2 * 32 + j % 2 * 8);
    __syncthreads();

    attend_f32x16_t o[kWide] = {};
    float top = -__builtin_inff(), total = 0.0f;
    uint32_t step, last;
    attend_split(a, at.longest, range, split, step, last);
    const uint32_t shift = a.s.page_shift, inside = (1u << shift) - 1;
    const uint32_t k_row = c / 4 % 2 * 16 + c / 8 * 4 + c % 4;
    AttendEntry k_entry[2], v_entry[2];
    const auto find_pages = [&](uint32_t at, uint32_t zero) {
        const auto entry_at = [&](uint32_t group) { return attend_ask(a.s, s, group >> shift, at < last && group < range.high && group + 16 > range.low); };
        if constexpr (WIDE) {
            k_entry[0] = k_entry[1] = v_entry[0] = v_entry[1] = attend_ask(a.s, s, __builtin_amdgcn_readfirstlane(at * kAttendStep >> shift), at < last, zero);
            return;
        }
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x) {
            const uint32_t k0 = at * kAttendStep + x * 32;
            k_entry[x] = entry_at(k0 + c / 4 % 2 * 16);
            v_entry[x] = entry_at(k0 + h * 16);
        }
    };
    uint4 k[2][kWide], v[2][kWide];
    float k_scale[2], v_scale[2];
    bool held[2];
    uint32_t found = 0;  // NaN among values that not all rows see
    const auto request_keys = [&](uint32_t at) {
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x) {
            const uint32_t k_page = attend_told<WIDE>(a.s, k_entry[x]);
            const uint64_t page = static_cast<uint64_t>(k_page != kNoPage ? k_page : 0) * a.c.heads + head;  // (read, and not used)
            const uint8_t *from = WIDE ? a.c.k + ((page << shift) + ((at * kAttendStep + x * 32) & inside)) * DIM + k_row * DIM + h * 16
                                       : a.c.k + ((page << shift) + ((at * kAttendStep + x * 32 + k_row) & inside)) * DIM + h * 16;
            k_scale[x] = a.c.k_scales[page];
#pragma unroll
            for (uint32_t j = 0; j < kWide; ++j)
                k[x][j] = *reinterpret_cast<const uint4 *>(from + j * 32);
        }
    };
    // (and the entries of the step `next`, before the values: whoever waits for them does not wait for these)
    const auto request_values = [&](uint32_t at, uint32_t next) {
        const uint32_t v_page[2] = {attend_told<WIDE>(a.s, v_entry[0]), attend_told<WIDE>(a.s, v_entry[1])};
        find_pages(next, attend_zero());
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x) {
            held[x] = v_page[x] != kNoPage;
            const uint64_t page = static_cast<uint64_t>(held[x] ? v_page[x] : 0) * a.c.heads + head;
            const uint8_t *from = WIDE ? a.c.v + (page * DIM << shift) + ((at * kAttendStep + x * 32) & inside) + (c << shift) + h * 16
                                       : a.c.v + ((page * DIM + c) << shift) + ((at * kAttendStep + x * 32 + h * 16) & inside);
            v_scale[x] = a.c.v_scales[page];
#pragma unroll
            for (uint32_t f = 0; f < kWide; ++f)
                v[x][f] = *reinterpret_cast<const uint4 *>(from + (f * 32 << shift));
        }
    };
    step += wave;
    const uint32_t begin = step;
    if (step < last) {
        find_pages(step, 0);
        request_keys(step);
        request_values(step, step + WAVES);
    }
    for (; step < last; step += WAVES) {
        const uint32_t k0 = step * kAttendStep;
        asm volatile("" ::: "memory");  // (the queries stay in LDS)
        attend_f32x16_t score[2] = {};
#pragma unroll
        for (uint32_t j = 0; j < kWide; ++j) {
            const attend_bf16x8_t first = queries[j * 2][lane], second = queries[j * 2 + 1][lane];
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x) {
                score[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(attend_widen(k[x][j].x, k[x][j].y, k_scale[x]), first, score[x], 0, 0, 0);
                score[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(attend_widen(k[x][j].z, k[x][j].w, k_scale[x]), second, score[x], 0, 0, 0);
            }
        }
        if (step + WAVES < last)
            request_keys(step + WAVES);
        if (attend_edge(range, k0) || __any(!held[0] || !held[1])) {
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x) {
                const uint32_t group = k0 + x * 32 + h * 16;
#pragma unroll
                for (uint32_t e = 0; e < 16; ++e)
                    if (!(held[x] && group + e >= my_low && group + e < my_high))
                        score[x][e] = -__builtin_inff();
                const int32_t from = held[x] ? static_cast<int32_t>(range.low - group) : 16, upto = held[x] ? static_cast<int32_t>(range.high - group) : 0;
                const uint32_t m0 = attend_bytes(from, upto, 0), m1 = attend_bytes(from, upto, 1), m2 = attend_bytes(from, upto, 2), m3 = attend_bytes(from, upto, 3);
#pragma unroll
                for (uint32_t f = 0; f < kWide; ++f)
                    found |= attend_clean(v[x][f].x, m0) | attend_clean(v[x][f].y, m1) | attend_clean(v[x][f].z, m2) | attend_clean(v[x][f].w, m3);
            }
        }
        float most = -__builtin_inff();
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x)
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e)
                most = fmaxf(most, score[x][e]);
        most = attend_max_of_halves(most) * a.scale;
        if (__any(most > top + kAttendSlack)) {
            const float higher = most > top + kAttendSlack ? most : top, less = higher == -__builtin_inff() ? 1.0f : attend_exp2(top - higher);
            top = higher;
            total *= less;
#pragma unroll
            for (uint32_t f = 0; f < kWide; ++f)
                o[f] *= less;
        }
        const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x) {
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) {
                score[x][e] = attend_exp2(score[x][e] * a.scale - base);
                total += score[x][e];
            }
            const attend_f32x16_t &w = score[x];
            const float of_values = held[x] ? v_scale[x] : 1.0f;
            const attend_bf16x8_t p0 = attend_round(w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
            const attend_bf16x8_t p1 = attend_round(w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]);
#pragma unroll
            for (uint32_t f = 0; f < kWide; ++f) {
                o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(attend_widen(v[x][f].x, v[x][f].y, of_values), p0, o[f], 0, 0, 0);
                o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(attend_widen(v[x][f].z, v[x][f].w, of_values), p1, o[f], 0, 0, 0);
            }
        }
        if (step + WAVES < last)
            request_values(step + WAVES, step + 2 * WAVES);
    }
    total += __shfl_xor(total, 32);
    if (__any(found != 0)) {
        // a row that sees a value that is NaN has it: products of where NaN is with who sees it
#pragma unroll
        for (uint32_t f = 0; f < kWide; ++f) {
            attend_f32x16_t seen = {};
            for (step = begin; step < last; step += WAVES)
                seen = attend_nans(a, s, head, DIM, f * 32 + c, step * kAttendStep, h, my_low, my_high, seen);
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e)
                o[f][e] = seen[e] > 0.0f ? __builtin_nanf("") : o[f][e];
        }
    }
    if (h == 0)
        stats[wave][c] = make_float2(top, total);
#pragma unroll
    for (uint32_t f = 0; f < kWide; ++f)
#pragma unroll
        for (uint32_t e = 0; e < 16; e += 4)
            *reinterpret_cast<float4 *>(&sums[wave][c][f * 32 + e * 2 + h * 4]) = make_float4(o[f][e], o[f][e + 1], o[f][e + 2], o[f][e + 3]);
    __syncthreads();
    attend_leave<DIM, WAVES, kAttendSomeRows>(a, n, head, split, row0, row_end, sums, stats);
}

// ---- many rows: a wave has 32 rows, a workgroup 128 or 256.  A step's keys and values are widened once, by all waves, into LDS, from where every wave reads
// them as operands; the next step's bytes are on their way meanwhile, and the pages of the one behind it.  Lanes hold keys as above.
// In LDS: row c of 32 of the keys' operand, its pieces of 16 bytes (8 features) in places p ^ c % 16 (rows of 128 bytes: p ^ c / 2 % 8); the values' row is
// a feature, 64 keys in 8 pieces, in places p ^ feature / 2 % 8: the sixteen lanes that read together, 0 to 3, 12 to 15, 20 to 27 or the others, find different banks.
// What bounds it: a step of a wave takes the matrix cores 1024 cycles (head_dim 128), the vector unit about 1450 (exponentials 512, the rest of the softmax
// 400, requests, widening and LDS addresses), LDS 320, for eight waves 2560; two waves share a SIMD.  A prompt of 4096 tokens, 32
// query heads on 8, takes 148 us with 256 rows to a workgroup (929 TFLOP/s), 159 with 128; one of 16384 2.08 ms, 1057 TFLOP/s.  Neither unit is full: of 4096 tokens the matrix
// cores are busy 0.36 of the launch and the vector unit issues 0.40 of it (16384: 0.44 and 0.46), with 1.74 (1.92) waves to a SIMD, which spend 0.32 of their time waiting, for
// LDS, for requests, and for each other at the barrier of a step, which keeps a workgroup's waves in one phase; 0.30 waiting for their turn at a unit that another one has.
// With 128 rows it would take 126 without widening into LDS, 149 without requests, 146 without exponentials.  Tried: a wave with 64 rows halves
// what LDS reads, but fills 400 registers and is alone on its SIMD, 350 us; the next step's products beside this step's exponentials in the program, 169 us, as
// 256 registers leave none for operands on their way; the rows' sums by dot products or in the matrix cores, 178 and 186;
// the workgroup's halves a phase apart, one at products while the other is at weights, with a barrier to each phase, 151 to 162 against 148 on the same card.
constexpr int kSchedVector = 0x2, kSchedMatrix = 0x8, kSchedLds = 0x100;  // kinds of instructions (sched_group_barrier)

template <uint32_t DIM, bool WIDE, uint32_t WAVES>
__global__ void __launch_bounds__(WAVES * 64, 2) attend_many_kernel(const AttendArgs a)
{
    constexpr uint32_t kPieces = DIM / 8, kBytes = kAttendStep * DIM * 2;
    constexpr uint32_t kRows = WAVES * 32, kItems = kAttendStep * DIM / 16 / (WAVES * 64);  // 16 bytes of the cache, of keys and of values, to a thread
    constexpr uint32_t kKeysApart = kAttendStep / kItems, kFeaturesApart = DIM / kItems;
    __shared__ __align__(16) uint8_t key_space[2][kBytes];
    __shared__ __align__(16) uint8_t value_space[2][kBytes];
    __shared__ uint4 there_space[2];  // of four times 16 keys: not 0 if they have a page
    const uint32_t head = blockIdx.x % a.c.heads, split = blockIdx.x / a.c.heads % a.splits, tile = a.tiles - 1 - blockIdx.x / a.c.heads / a.splits;
    const Found at = find_sequence(a.s, a.numbers, tile, a.splits > 1);
    if (at.s >= a.s.count)
        return;
    const uint32_t s = at.s;
    const NewTokens n = at.n;
    const uint64_t row0_wide = at.tile * kRows;
    const uint32_t rows = n.count * a.group;
    if (row0_wide >= rows)
        return;
    const uint32_t row0 = static_cast<uint32_t>(row0_wide), row_end = rows - row0 < kRows ? rows : row0 + kRows;
    const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64, c = lane % 32, h = lane / 32;
    const AttendRange range = attend_range(n, row0 / a.group, (row_end - 1) / a.group, a.window);
    uint32_t begin, last;
    attend_split(a, at.longest, range, split, begin, last);

    // the wave's rows, and the lane's
    const uint32_t wave0 = row0 + wave * 32 < row_end ? row0 + wave * 32 : row_end - 1, wave_end = wave0 + 32 < row_end ? wave0 + 32 : row_end;
    const AttendRange of_wave = attend_range(n, wave0 / a.group, (wave_end - 1) / a.group, a.window);
    const bool mine = row0 + wave * 32 + c < row_end;
    const uint32_t row = mine ? row0 + wave * 32 + c : row_end - 1, behind = n.first + row / a.group + 1;
    const uint32_t my_high = mine ? behind : 0, my_low = a.window && behind > a.window ? behind - a.window : 0;
    attend_bf16x8_t q[DIM / 16];
    const uint16_t *q_at = a.q + (n.begin + row / a.group) * a.q_row + (head * a.group + row % a.group) * DIM + h * 8;
#pragma unroll
    for (uint32_t j = 0; j < DIM / 16; ++j)
        q[j] = *reinterpret_cast<const attend_bf16x8_t *>(q_at + j * 16);

    // the thread's items of a step: a key's 16 features, a feature's 16 keys
    const uint32_t shift = a.s.page_shift, inside = (1u << shift) - 1;
    const uint32_t k_key = threadIdx.x / (DIM / 16), k_part = threadIdx.x % (DIM / 16), v_feature = threadIdx.x / 4, v_part = threadIdx.x % 4;
    AttendEntry k_entry[WIDE ? 1 : kItems], v_entry;
    const auto find_key_pages = [&](uint32_t at, uint32_t zero) {
#pragma unroll
        for (uint32_t i = 0; i < (WIDE ? 1 : kItems); ++i)
            k_entry[i] = attend_ask(a.s, s, (at * kAttendStep + (WIDE ? 0 : k_key + i * kKeysApart)) >> shift, at < last, zero);
    };
    const auto find_value_pages = [&](uint32_t at) {
        const uint32_t v0 = at * kAttendStep + (WIDE ? 0 : v_part * 16);
        if constexpr (WIDE)
            v_entry = k_entry[0];
        else
            v_entry = attend_ask(a.s, s, v0 >> shift, at < last && v0 < range.high && v0 + 16 > range.low);
    };
    uint4 k_item[kItems], v_item[kItems];
    float k_scale[WIDE ? 1 : kItems], v_scale;
    bool k_there[WIDE ? 1 : kItems], v_there;
    const auto request_keys = [&](uint32_t at) {
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t p = WIDE ? 0 : i;
            const uint32_t k_page = attend_told<WIDE>(a.s, k_entry[p]);
            k_there[p] = k_page != kNoPage;
            const uint64_t page = static_cast<uint64_t>(k_there[p] ? k_page : 0) * a.c.heads + head;  // (read, and not used)
            k_scale[p] = a.c.k_scales[page];
            const uint8_t *from = a.c.k + ((page << shift) + ((at * kAttendStep + (WIDE ? 0 : k_key + i * kKeysApart)) & inside)) * DIM;
            k_item[i] = *reinterpret_cast<const uint4 *>(from + (WIDE ? (k_key + i * kKeysApart) * DIM : 0) + k_part * 16);
        }
    };
    const auto request_values = [&](uint32_t at) {
        const uint32_t v_page = attend_told<WIDE>(a.s, v_entry);
        v_there = v_page != kNoPage;
        const uint64_t page = static_cast<uint64_t>(v_there ? v_page : 0) * a.c.heads + head;
        v_scale = a.c.v_scales[page];
        const uint8_t *from = a.c.v + (page * DIM << shift) + ((at * kAttendStep + (WIDE ? 0 : v_part * 16)) & inside);
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i)
            v_item[i] = *reinterpret_cast<const uint4 *>(from + ((v_feature + i * kFeaturesApart) << shift) + (WIDE ? v_part * 16 : 0));
    };
    const auto put_keys = [&](uint32_t turn) {
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t p = WIDE ? 0 : i, key = k_key + i * kKeysApart, x = key % 32, r = key / 32 * 32 + x / 4 % 4 * 8 + x / 16 * 4 + x % 4;
            const uint32_t turned = r / (16 / kPieces) % kPieces;
            uint8_t *line = key_space[turn] + r * DIM * 2;
            *reinterpret_cast<attend_bf16x8_t *>(line + ((k_part * 2) ^ turned) * 16) = attend_widen(k_item[i].x, k_item[i].y, k_scale[p]);
            *reinterpret_cast<attend_bf16x8_t *>(line + ((k_part * 2 + 1) ^ turned) * 16) = attend_widen(k_item[i].z, k_item[i].w, k_scale[p]);
            if (!WIDE && k_part == 0 && key % 16 == 0)
                reinterpret_cast<uint32_t *>(&there_space[turn])[key / 16] = k_there[p];
        }
        if (WIDE && threadIdx.x == 0)
            there_space[turn] = make_uint4(k_there[0], k_there[0], k_there[0], k_there[0]);
    };
    uint32_t found = 0;  // NaN among values that not all rows see
    const auto put_values = [&](uint32_t at, uint32_t turn) {
        if (attend_edge(range, at * kAttendStep) || __any(!v_there)) {
            // values that not all rows see: those that none does, and NaN (0 * NaN is), are made 0; who sees NaN is looked up in the end
            const uint32_t v0 = at * kAttendStep + v_part * 16;
            const int32_t from = v_there ? static_cast<int32_t>(range.low - v0) : 16, upto = v_there ? static_cast<int32_t>(range.high - v0) : 0;
#pragma unroll
            for (uint32_t i = 0; i < kItems; ++i) {
                found |= attend_clean(v_item[i].x, attend_bytes(from, upto, 0)) | attend_clean(v_item[i].y, attend_bytes(from, upto, 1));
                found |= attend_clean(v_item[i].z, attend_bytes(from, upto, 2)) | attend_clean(v_item[i].w, attend_bytes(from, upto, 3));
            }
        }
        const float of_values = v_there ? v_scale : 1.0f;
#pragma unroll
        for (uint32_t i = 0; i < kItems; ++i) {
            const uint32_t feature = v_feature + i * kFeaturesApart;
            uint8_t *line = value_space[turn] + feature * kAttendStep * 2;
            *reinterpret_cast<attend_bf16x8_t *>(line + ((v_part * 2) ^ (feature / 2 % 8)) * 16) = attend_widen(v_item[i].x, v_item[i].y, of_values);
            *reinterpret_cast<attend_bf16x8_t *>(line + ((v_part * 2 + 1) ^ (feature / 2 % 8)) * 16) = attend_widen(v_item[i].z, v_item[i].w, of_values);
        }
    };

    attend_f32x16_t o[DIM / 32] = {};
    float top = -__builtin_inff(), total = 0.0f, most = 0.0f;
    const auto products = [&](attend_f32x16_t (&score)[2], uint32_t turn) {
#pragma unroll
        for (uint32_t j = 0; j < DIM / 16; ++j)
#pragma unroll
            for (uint32_t half = 0; half < 2; ++half) {
                const attend_bf16x8_t keys = *reinterpret_cast<const attend_bf16x8_t *>(key_space[turn] + (half * 32 + c) * DIM * 2 +
                                                                                        ((j * 2 + h) ^ (c / (16 / kPieces) % kPieces)) * 16);
                score[half] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys, q[j], j ? score[half] : attend_f32x16_t{}, 0, 0, 0);
            }
    };
    // what the rows do not see, and their maxima
    const auto look = [&](attend_f32x16_t (&score)[2], uint32_t at, uint32_t turn) {
        const uint4 there = there_space[turn];
        const uint32_t k0 = at * kAttendStep;
        if (attend_edge(of_wave, k0) || __builtin_amdgcn_readfirstlane(there.x & there.y & there.z & there.w) == 0) {
            asm volatile("");  // (a branch around it, not 130 instructions of every step)
            const uint32_t have[2] = {h ? there.y : there.x, h ? there.w : there.z};
#pragma unroll
            for (uint32_t half = 0; half < 2; ++half)
#pragma unroll
                for (uint32_t e = 0; e < 16; ++e) {
                    const uint32_t key = k0 + half * 32 + h * 16 + e;
                    if (!(key >= my_low && key < my_high && have[half]))
                        score[half][e] = -__builtin_inff();
                }
        }
        most = -__builtin_inff();
#pragma unroll
        for (uint32_t half = 0; half < 2; ++half)
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e)
                most = fmaxf(most, score[half][e]);
        most = attend_max_of_halves(most) * a.scale;
    };
    if (begin < last) {
        find_key_pages(begin, 0);
        find_value_pages(begin);
        request_keys(begin);
        request_values(begin);
        find_key_pages(begin + 1, attend_zero());
        find_value_pages(begin + 1);
        put_keys(0);
        put_values(begin, 0);
    }
#pragma unroll
    for (uint32_t j = 0; j < DIM / 16; ++j)
        asm volatile("" ::"v"(q[j]));  // (the queries are waited for here, not in every step)
    uint32_t step = begin;
    for (uint32_t turn = 0; step < last; ++step, turn ^= 1) {
        __syncthreads();
        if (step + 1 < last) {
            request_keys(step + 1);
            request_values(step + 1);
            find_key_pages(step + 2, attend_zero());
            find_value_pages(step + 2);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        attend_f32x16_t now[2];
        products(now, turn);
        // (six operands on their way from LDS before the first product, one more behind each)
        __builtin_amdgcn_sched_group_barrier(kSchedLds, 6, 0);
#pragma unroll
        for (uint32_t g = 0; g < DIM / 8 - 6; ++g) {
            __builtin_amdgcn_sched_group_barrier(kSchedMatrix, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kSchedMatrix, 6, 0);
        __builtin_amdgcn_sched_barrier(0);
        look(now, step, turn);
        if (__any(most > top + kAttendSlack)) {
            const float higher = most > top + kAttendSlack ? most : top, less = higher == -__builtin_inff() ? 1.0f : attend_exp2(top - higher);
            top = higher;
            total *= less;
#pragma unroll
            for (uint32_t f = 0; f < DIM / 32; ++f)
                o[f] *= less;
        }
        const float base = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            attend_f32x16_t &w = now[u / 2];
            const uint32_t e = u % 2 * 8;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                w[e + i] = attend_exp2(w[e + i] * a.scale - base);
                total += w[e + i];
            }
            const attend_bf16x8_t p = attend_round(w[e], w[e + 1], w[e + 2], w[e + 3], w[e + 4], w[e + 5], w[e + 6], w[e + 7]);
#pragma unroll
            for (uint32_t f = 0; f < DIM / 32; ++f) {
                const attend_bf16x8_t values = *reinterpret_cast<const attend_bf16x8_t *>(value_space[turn] + (f * 32 + c) * kAttendStep * 2 +
                                                                                          ((u / 2 * 4 + h * 2 + u % 2) ^ (c / 2 % 8)) * 16);
                o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values, p, o[f], 0, 0, 0);
            }
        }
        // Pages of less than a step, heads of 128: four operands before the exponentials; then the products, the remaining exponentials between them (4096
        // tokens of 32 heads on 8 in pages of 16: 160 us, in the compiler's order 168).  Elsewhere its order is the better one (pages of 64: 4096 tokens 159 us,
        // this one 161; 16384 tokens 2140 and 2290).
        if constexpr (!WIDE && DIM > 64) {
            __builtin_amdgcn_sched_group_barrier(kSchedLds, 4, 1);
            __builtin_amdgcn_sched_group_barrier(kSchedVector, 34, 1);
#pragma unroll
            for (uint32_t g = 0; g < DIM / 8 - 4; ++g) {
                __builtin_amdgcn_sched_group_barrier(kSchedMatrix, 1, 1);
                __builtin_amdgcn_sched_group_barrier(kSchedLds, 1, 1);
                __builtin_amdgcn_sched_group_barrier(kSchedVector, 8, 1);
            }
            __builtin_amdgcn_sched_group_barrier(kSchedMatrix, 4, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        // (widening and the next requests go before the products of the other workgroup's wave on the SIMD: 159 us, without that 163)
        __builtin_amdgcn_s_setprio(1);
        if (step + 1 < last) {
            put_keys(turn ^ 1);
            put_values(step + 1, turn ^ 1);
        }
    }
    total += __shfl_xor(total, 32);
    if (__syncthreads_or(found != 0)) {
        // a row that sees a value that is NaN has it: products of where NaN is with who sees it
#pragma unroll
        for (uint32_t f = 0; f < DIM / 32; ++f) {
            attend_f32x16_t seen = {};
            for (step = begin; step < last; ++step)
                seen = attend_nans(a, s, head, DIM, f * 32 + c, step * kAttendStep, h, my_low, my_high, seen);
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e)
                o[f][e] = seen[e] > 0.0f ? __builtin_nanf("") : o[f][e];
        }
    }
    if (!mine)
        return;
    const uint64_t to = attend_row(a, n, head, row);
    if (a.splits > 1) {
        const uint64_t place = static_cast<uint64_t>(split) * a.s.rows * a.q_heads + to;
        if (h == 0)
            a.stats[place] = make_float2(top, total);
#pragma unroll
        for (uint32_t f = 0; f < DIM / 32; ++f)
#pragma unroll
            for (uint32_t e = 0; e < 16; e += 4)
                *reinterpret_cast<float4 *>(a.partial + place * DIM + f * 32 + e * 2 + h * 4) = make_float4(o[f][e], o[f][e + 1], o[f][e + 2], o[f][e + 3]);
        return;
    }
    const float once = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (uint32_t f = 0; f < DIM / 32; ++f)
#pragma unroll
        for (uint32_t e = 0; e < 16; e += 4) {
            typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
            const attend_f32x4_t v = {o[f][e] * once, o[f][e + 1] * once, o[f][e + 2] * once, o[f][e + 3] * once};
            *reinterpret_cast<bf16x4_t *>(a.out + to * DIM + f * 32 + e * 2 + h * 4) = __builtin_convertvector(v, bf16x4_t);
        }
}

// The splits of a row together; four features to a lane, and GROUPS of lanes with every GROUPS-th split each.
template <uint32_t DIM, uint32_t GROUPS>
__global__ void __launch_bounds__(kAttendThreads) attend_join_kernel(const AttendArgs a)
{
    constexpr uint32_t kLanes = DIM / 4, kRows = kAttendThreads / kLanes / GROUPS;
    const uint64_t count = static_cast<uint64_t>(a.s.rows) * a.q_heads;
    const uint32_t group = threadIdx.x / kLanes % GROUPS, in_rows = threadIdx.x / (kLanes * GROUPS);
    const uint64_t row = static_cast<uint64_t>(blockIdx.x) * kRows + in_rows;
    const uint32_t at = threadIdx.x % kLanes * 4;
    const int64_t token = static_cast<int64_t>(row / a.q_heads);
    const bool here = row < count && token >= a.s.starts[0] && token < a.s.starts[a.s.count];  // (others are nobody's)
    float all = -__builtin_inff(), whole = 0.0f;
    attend_f32x4_t sum = {};
    if (here) {
        const float2 *stats = a.stats + row;
        const float *partial = a.partial + row * DIM + at;
#pragma unroll 4
        for (uint32_t p = group; p < a.splits; p += GROUPS)
            all = fmaxf(all, stats[p * count].x);
        const float base = all == -__builtin_inff() ? 0.0f : all;
#pragma unroll 4
        for (uint32_t p = group; p < a.splits; p += GROUPS) {
            const float2 part = stats[p * count];
            const float share = attend_exp2(part.x - base);
            whole += share * part.y;
            sum += share * *reinterpret_cast<const attend_f32x4_t *>(partial + p * count * DIM);
        }
    }
    if constexpr (GROUPS > 1) {
        __shared__ attend_f32x4_t sums[GROUPS][kRows * kLanes];
        __shared__ float2 parts[GROUPS][kRows * kLanes];
        const uint32_t place = in_rows * kLanes + threadIdx.x % kLanes;
        sums[group][place] = sum;
        parts[group][place] = make_float2(all, whole);
        __syncthreads();
        if (group)
            return;
#pragma unroll
        for (uint32_t other = 1; other < GROUPS; ++other)
            all = fmaxf(all, parts[other][place].x);
        const float base = all == -__builtin_inff() ? 0.0f : all;
        sum = {};
        whole = 0.0f;
#pragma unroll
        for (uint32_t other = 0; other < GROUPS; ++other) {
            const float share = attend_exp2(parts[other][place].x - base);
            whole += share * parts[other][place].y;
            sum += share * sums[other][place];
        }
    }
    if (!here)
        return;
    typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
    sum *= whole == 0.0f ? 0.0f : 1.0f / whole;
    *reinterpret_cast<bf16x4_t *>(a.out + row * DIM + at) = __builtin_convertvector(sum, bf16x4_t);
}

}  // namespace nz
