// Keys and values into a cache of 8-bit values for gfx950: rotated to their positions, scaled by a power of two for each page and head, rounded.
//
// A workgroup has one page that new tokens go to, one head, and its keys or its values: it finds the largest of the new values, sets the scale, and
// writes the bytes.  Memory bounds it (4 bytes read and 1 written a value, 8 operations); a decoding batch, whose workgroups have one
// token each, is bound by the launch and a chain of four reads: whose tile, which rows, which page, the values.  Measured, 8 heads of 128 and 32 query heads in
// float32: 3323 tokens of two prompts 20.2 us (124 MB, 6.1 TB/s), one token each of 48 sequences 7.0 us.
// Values lie feature by feature in a page, so that the attention kernel finds consecutive tokens of a feature side by side; their bytes go
// through LDS to be turned.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "neuzip_sequences.h"

namespace nz {

constexpr uint32_t kAppendThreads = 256;
constexpr float kE4m3Most = 448.0f;
constexpr int kLeastScale = -100;  // exponent

struct CacheView {
    uint8_t *k, *v;
    float *k_scales, *v_scales;
    uint32_t heads;
};

struct AppendArgs {
    SequencesView s;
    CacheView c;
    const void *k, *v, *q;
    uint64_t k_row, v_row, q_row;
    uint16_t *q_out;
    const float *rotary;
    uint32_t q_heads;
    uint32_t tiles;  // workgroups: tiles * heads * 2, and behind them one for each row of q
};

// The sequence that a tile of number `id` is in.
struct Found {
    uint32_t s;          // the last in 0 .. count - 1 with first_tile(s) <= id; count if there is none
    NewTokens n;
    uint64_t tile;       // id, counted from the sequence's first
    uint32_t longest;    // no sequence has more tokens
};

// A wave works it out together.  Up to 64 sequences are all read at once, so that what comes next waits for memory once.
__device__ __forceinline__ Found find_sequence(const SequencesView &v, const TileNumbers &t, uint64_t id, bool with_longest)
{
    const uint32_t lane = threadIdx.x % 64;
    Found f;
    int32_t longest = 0;
    if (v.count <= 64) {
        const uint32_t at = lane < v.count ? lane : v.count - 1;
        const int32_t begin = v.starts[at], end = v.starts[at + 1], length = v.lengths[at];
        const uint32_t before = __popcll(__ballot(lane < v.count && first_tile(t, begin, lane) <= id));
        f.s = before ? before - 1 : v.count;
        const uint32_t from = __builtin_amdgcn_readfirstlane(before ? before - 1 : 0);
        f.n = new_tokens(v, __builtin_amdgcn_readlane(begin, from), __builtin_amdgcn_readlane(end, from), __builtin_amdgcn_readlane(length, from));
        const uint64_t first = first_tile(t, __builtin_amdgcn_readlane(begin, from), from);
        if (first > id)  // (starts that do not ascend)
            f.s = v.count;
        f.tile = id - first;
        longest = length;
    } else {
        uint32_t base = 0, left = v.count;
        while (left > 1) {
            const uint32_t step = (left + 63) / 64, at = base + lane * step;
            const bool before = lane * step < left && first_tile(t, v.starts[at], at) <= id;
            const uint32_t last = __popcll(__ballot(before));
            if (last == 0) {
                f.s = v.count;
                return f;
            }
            base += (last - 1) * step;
            left -= (last - 1) * step;
            left = left < step ? left : step;
        }
        f.n = new_tokens(v, base);
        const uint64_t first = first_tile(t, v.starts[base], base);
        f.s = first <= id ? base : v.count;
        f.tile = id - first;
        if (with_longest)
            for (uint32_t s = lane; s < v.count; s += 64)
                longest = max(longest, v.lengths[s]);
    }
    if (with_longest) {
#pragma unroll
        for (int apart = 32; apart; apart >>= 1)
            longest = max(longest, __shfl_xor(longest, apart));
        f.longest = __builtin_amdgcn_readfirstlane(longest > 0 ? static_cast<uint32_t>(longest) : 0);
    }
    // (every lane has the same; what hangs on it is scalar once that is said)
    f.s = __builtin_amdgcn_readfirstlane(f.s);
    f.n.begin = __builtin_amdgcn_readfirstlane(f.n.begin);
    f.n.count = __builtin_amdgcn_readfirstlane(f.n.count);
    f.n.first = __builtin_amdgcn_readfirstlane(f.n.first);
    f.n.length = __builtin_amdgcn_readfirstlane(f.n.length);
    f.tile = static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(f.tile >> 32))) << 32 |
             __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(f.tile));
    return f;
}

__device__ __forceinline__ void append_load(const float *from, float (&v)[8])
{
    const float4 a = reinterpret_cast<const float4 *>(from)[0], b = reinterpret_cast<const float4 *>(from)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void append_load(const uint16_t *from, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(from);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[2 * i] = __builtin_bit_cast(float, w[i] << 16), v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
}

// x[i], x[i + D / 2] by the angle's cosine and sine.  Products and sums rounded one by one, as the formula has them.
__device__ __forceinline__ void append_rotate(const float *angle, uint32_t half, float (&a)[8], float (&b)[8])
{
#pragma clang fp contract(off)
    float cos[8], sin[8];
    append_load(angle, cos);
    append_load(angle + half, sin);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = a[i], y = b[i];
        a[i] = x * cos[i] - y * sin[i];
        b[i] = y * cos[i] + x * sin[i];
    }
}

// The least power of two from 2^-100 on by which `most`, a finite number, is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ float append_scale(float most)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, most);
    const int e = static_cast<int>(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
    return __builtin_bit_cast(float, static_cast<uint32_t>((e > kLeastScale ? e : kLeastScale) + 127) << 23);
}
__device__ __forceinline__ float append_finite(float v)
{
    const float m = fabsf(v);
    return m < __builtin_inff() ? m : 0.0f;
}
__device__ __forceinline__ float append_clamp(float v) { return v != v ? v : fminf(fmaxf(v, -kE4m3Most), kE4m3Most); }
__device__ __forceinline__ uint32_t append_code(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(append_clamp(a), append_clamp(b), 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(append_clamp(c), append_clamp(d), w, true));
}
// four bytes, each rounded to a scale that is larger by 1 / ratio
__device__ __forceinline__ uint32_t append_again(uint32_t w, float ratio)
{
    return append_code(__builtin_amdgcn_cvt_f32_fp8(w, 0) * ratio, __builtin_amdgcn_cvt_f32_fp8(w, 1) * ratio, __builtin_amdgcn_cvt_f32_fp8(w, 2) * ratio,
                       __builtin_amdgcn_cvt_f32_fp8(w, 3) * ratio);
}

// The queries of one row.
template <class T>
__device__ __forceinline__ void append_queries(const AppendArgs &a, uint32_t row, uint32_t dim)
{
    const Found found = find_sequence(a.s, {0, 1, 0}, row, false);
    const NewTokens n = found.n;
    if (found.s >= a.s.count || found.tile >= n.count)
        return;  // behind the last sequence
    const uint32_t half = dim / 2, pieces = half / 8;
    const T *q = static_cast<const T *>(a.q) + row * a.q_row;
    const float *angle = a.rotary ? a.rotary + static_cast<uint64_t>(n.first + (row - n.begin)) * dim : nullptr;
    uint16_t *out = a.q_out + static_cast<uint64_t>(row) * a.q_heads * dim;
    for (uint32_t i = threadIdx.x; i < a.q_heads * pieces; i += kAppendThreads) {
        const uint32_t head = i / pieces, at = i % pieces * 8;
        float x[8] = {}, y[8] = {};
        if (n.length) {
            append_load(q + head * dim + at, x);
            append_load(q + head * dim + half + at, y);
            if (angle)
                append_rotate(angle + at, half, x, y);
        }
        typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
        typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8_t;
        const f32x8_t fx = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}, fy = {y[0], y[1], y[2], y[3], y[4], y[5], y[6], y[7]};
        *reinterpret_cast<uint4 *>(out + head * dim + at) = __builtin_bit_cast(uint4, __builtin_convertvector(fx, bf16x8_t));
        *reinterpret_cast<uint4 *>(out + head * dim + half + at) = __builtin_bit_cast(uint4, __builtin_convertvector(fy, bf16x8_t));
    }
}

// DIM * page_tokens <= ITEMS * 16 * kAppendThreads
template <class T, uint32_t DIM, uint32_t ITEMS>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs a)
{
    constexpr uint32_t kHalf = DIM / 2, kPieces = kHalf / 8;  // an item: eight values of a token's first half and the eight that turn with them
    constexpr uint32_t kMostTokens = ITEMS * 16 * kAppendThreads / DIM;
    __shared__ float most_of[kAppendThreads / 64];
    __shared__ __align__(16) uint8_t turned[DIM * (kMostTokens + 4)];
    const uint32_t kv_wgs = a.tiles * a.c.heads * 2;
    if (blockIdx.x >= kv_wgs) {
        append_queries<T>(a, blockIdx.x - kv_wgs, DIM);
        return;
    }
    const uint32_t shift = a.s.page_shift, size = 1u << shift;
    const uint32_t tile = blockIdx.x / (a.c.heads * 2), head = blockIdx.x / 2 % a.c.heads;
    const bool values = blockIdx.x % 2;
    const Found found = find_sequence(a.s, {shift, 1, 2}, tile, false);
    if (found.s >= a.s.count)
        return;
    const NewTokens n = found.n;
    const uint64_t number_wide = (n.first >> shift) + found.tile;
    if (n.length == 0 || number_wide > (n.length - 1) >> shift)
        return;
    const uint32_t number = static_cast<uint32_t>(number_wide);
    const uint32_t page = page_of(a.s, found.s, number);
    if (page == kNoPage)
        return;
    // the new tokens' places in the page: begin .. end - 1
    const uint32_t base = number << shift;
    const uint32_t begin = n.first > base ? n.first - base : 0, end = n.length - base < size ? n.length - base : size;
    const uint32_t row0 = n.begin + (base + begin - n.first), items = (end - begin) * kPieces;
    const T *from = static_cast<const T *>(values ? a.v : a.k);
    const uint64_t row_elems = values ? a.v_row : a.k_row;
    const bool rotate = !values && a.rotary;
    float x[ITEMS][8], y[ITEMS][8];
    float most = 0.0f;
#pragma unroll
    for (uint32_t j = 0; j < ITEMS; ++j) {
        const uint32_t item = j * kAppendThreads + threadIdx.x;
        if (item < items) {
            const uint32_t token = item / kPieces, at = item % kPieces * 8;
            const T *p = from + (row0 + token) * row_elems + head * DIM + at;
            append_load(p, x[j]);
            append_load(p + kHalf, y[j]);
            if (rotate)
                append_rotate(a.rotary + static_cast<uint64_t>(base + begin + token) * DIM + at, kHalf, x[j], y[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                most = fmaxf(most, fmaxf(append_finite(x[j][i]), append_finite(y[j][i])));
        }
    }
    float *scale_at = (values ? a.c.v_scales : a.c.k_scales) + static_cast<uint64_t>(page) * a.c.heads + head;
    const float held = begin ? *scale_at : 0.0f;
#pragma unroll
    for (int apart = 32; apart; apart >>= 1)
        most = fmaxf(most, __shfl_xor(most, apart));
    if (threadIdx.x % 64 == 0)
        most_of[threadIdx.x / 64] = most;
    __syncthreads();
#pragma unroll
    for (uint32_t w = 0; w < kAppendThreads / 64; ++w)
        most = fmaxf(most, most_of[w]);
    const float fits = append_scale(most), scale = fmaxf(fits, held), inverse = 1.0f / scale;
    const bool grows = begin && scale > held;
    const float ratio = held * inverse;
    if (threadIdx.x == 0)
        *scale_at = scale;
    uint8_t *to = (values ? a.c.v : a.c.k) + ((static_cast<uint64_t>(page) * a.c.heads + head) * DIM << shift);
    if (!values) {
        if (grows)
            for (uint32_t i = threadIdx.x; i < begin * (DIM / 4); i += kAppendThreads) {
                uint32_t *w = reinterpret_cast<uint32_t *>(to) + i;
                *w = append_again(*w, ratio);
            }
#pragma unroll
        for (uint32_t j = 0; j < ITEMS; ++j) {
            const uint32_t item = j * kAppendThreads + threadIdx.x;
            if (item < items) {
                uint8_t *at = to + (begin + item / kPieces) * DIM + item % kPieces * 8;
                const float(&u)[8] = x[j], (&w)[8] = y[j];
                *reinterpret_cast<uint2 *>(at) = make_uint2(append_code(u[0] * inverse, u[1] * inverse, u[2] * inverse, u[3] * inverse),
                                                            append_code(u[4] * inverse, u[5] * inverse, u[6] * inverse, u[7] * inverse));
                *reinterpret_cast<uint2 *>(at + kHalf) = make_uint2(append_code(w[0] * inverse, w[1] * inverse, w[2] * inverse, w[3] * inverse),
                                                                    append_code(w[4] * inverse, w[5] * inverse, w[6] * inverse, w[7] * inverse));
            }
        }
        return;
    }
    const uint32_t stride = size + 4;
#pragma unroll
    for (uint32_t j = 0; j < ITEMS; ++j) {
        const uint32_t item = j * kAppendThreads + threadIdx.x;
        if (item < items) {
            uint8_t *at = turned + item % kPieces * 8 * stride + begin + item / kPieces;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const uint32_t u = append_code(x[j][i] * inverse, x[j][i + 1] * inverse, x[j][i + 2] * inverse, x[j][i + 3] * inverse);
                const uint32_t w = append_code(y[j][i] * inverse, y[j][i + 1] * inverse, y[j][i + 2] * inverse, y[j][i + 3] * inverse);
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    at[(i + b) * stride] = static_cast<uint8_t>(u >> 8 * b);
                    at[(kHalf + i + b) * stride] = static_cast<uint8_t>(w >> 8 * b);
                }
            }
        }
    }
    __syncthreads();
    // words of four tokens' bytes; what is not new in them stays, rounded anew if the scale grew
    const uint32_t first_word = grows ? 0 : begin / 4, words = (end + 3) / 4 - first_word;
    for (uint32_t i = threadIdx.x; i < DIM * words; i += kAppendThreads) {
        const uint32_t feature = i / words, slot = (first_word + i % words) * 4;
        uint32_t *at = reinterpret_cast<uint32_t *>(to + (feature << shift) + slot);
        const uint32_t coded = *reinterpret_cast<const uint32_t *>(turned + feature * stride + slot);
        uint32_t word = coded;
        if (slot < begin || slot + 4 > end) {
            const uint32_t there = *at, again = grows ? append_again(there, ratio) : there;
            word = 0;
#pragma unroll
            for (uint32_t b = 0; b < 4; ++b) {
                const uint32_t from_word = slot + b < begin ? again : slot + b < end ? coded : there;
                word |= from_word & (0xFFu << 8 * b);
            }
        }
        *at = word;
    }
}

}  // namespace nz
