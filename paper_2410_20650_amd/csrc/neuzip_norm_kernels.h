// Root-mean-square norm with the residual's addition, and its backward pass, for gfx950.
//
//   forward    t = T(x + r),  y = bf16(t * n * w),  n = 1 / sqrt(mean(t^2) + eps)
//   backward   g = dy * w,  dx = dt + n * (g - t * n^2 * mean(g * t)),  dw = sum over the tokens of dy * t * n
//
// Nothing is computed that a byte of memory would not pay for (about 6 and 16 operations an element), so memory bounds both: a row is read
// once and stays in registers, eight elements (a piece of 16 or 32 bytes) to a lane and request, between the sums and the results.
// THREADS lanes share a row: a wave where the rows are short or many, so that its sums need neither LDS nor a barrier; else a workgroup.
// The backward pass keeps w and the lane's part of dw in registers over all rows that a workgroup takes; the parts of a workgroup's rows
// are added in LDS, those of the workgroups by a launch of its own, in order, so that dw is the same every time.
// Measured, float32 results onto a bf16 stream of width 4096: 4096 tokens 27.4 us from memory (168 MB, 6.1 TB/s), 2048 tokens 15.6, their backward pass 16.0 (67 MB and
// 4 MB of parts, 4.5 TB/s) and 4.0 for the parts; one token 2.5 us, a launch.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

namespace nz {

constexpr uint32_t kNormThreads = 256;       // a workgroup of the forward pass with rows of up to 256 lanes
constexpr uint32_t kNormBackThreads = 1024;  // and of the backward pass: one on a CU
constexpr uint32_t kNormMostWgs = 256;       // of the backward pass, so many parts of dw
constexpr uint32_t kNormJoinColumns = 16;

struct NormArgs {
    const void *x, *residual;
    void *total;
    const float *weight;
    uint16_t *y;
    uint32_t tokens, width;
    float eps, per_width;
};

struct NormBackArgs {
    const void *total;
    const float *weight;
    const uint16_t *grad_y, *grad_total;
    uint16_t *grad_x;
    float *grad_weight;  // of one workgroup after the other, `width` floats each
    uint32_t tokens, width;
    float eps, per_width;
};

__device__ __forceinline__ uint32_t norm_pack(float a, float b)
{
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
    typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}
__device__ __forceinline__ float norm_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float norm_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }

// ---- eight consecutive elements: float or (uint16_t) bf16
__device__ __forceinline__ void norm_load(const float *from, float (&v)[8])
{
    const float4 a = reinterpret_cast<const float4 *>(from)[0], b = reinterpret_cast<const float4 *>(from)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void norm_load(const uint16_t *from, float (&v)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(from);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[2 * i] = norm_low(w[i]), v[2 * i + 1] = norm_high(w[i]);
}
__device__ __forceinline__ void norm_store(float *to, const float (&v)[8])
{
    reinterpret_cast<float4 *>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void norm_store(uint16_t *to, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(to) = make_uint4(norm_pack(v[0], v[1]), norm_pack(v[2], v[3]), norm_pack(v[4], v[5]), norm_pack(v[6], v[7]));
}
// what a value is once it is held in that type
__device__ __forceinline__ float norm_held(const float *, float v) { return v; }
__device__ __forceinline__ float norm_held(const uint16_t *, float v) { return norm_low(norm_pack(v, v)); }

__device__ __forceinline__ float norm_wave_sum(float v)
{
#pragma unroll
    for (int apart = 32; apart; apart >>= 1)
        v += __shfl_xor(v, apart);
    return v;
}

// The sum of v over the THREADS lanes of a row; every thread of the workgroup comes by.  space: a float for each wave, not in use by a
// sum that some wave may still be reading.
template <int THREADS>
__device__ __forceinline__ float norm_row_sum(float v, float *space)
{
    v = norm_wave_sum(v);
    if constexpr (THREADS > 64) {
        const uint32_t wave = threadIdx.x / 64;
        if (threadIdx.x % 64 == 0)
            space[wave] = v;
        __syncthreads();
        const uint32_t first = wave / (THREADS / 64) * (THREADS / 64);
        v = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < THREADS / 64; ++i)
            v += space[first + i];
    }
    return v;
}

template <int THREADS, int PIECES, class X, bool STREAM, class T>
__global__ void __launch_bounds__(THREADS > (int)kNormThreads ? THREADS : (int)kNormThreads) norm_kernel(const NormArgs a)
{
    __shared__ float space[16];
    const uint32_t row = blockIdx.x * (blockDim.x / THREADS) + threadIdx.x / THREADS, lane = threadIdx.x % THREADS;
    const bool here = row < a.tokens;
    const uint64_t at = static_cast<uint64_t>(here ? row : 0) * a.width;
    const X *x = static_cast<const X *>(a.x) + at;
    const T *residual = static_cast<const T *>(a.residual) + at;
    T *total = static_cast<T *>(a.total) + at;
    float t[PIECES][8];
    float squares = 0.0f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const uint32_t col = (p * THREADS + lane) * 8;
        if (col < a.width && here) {
            norm_load(x + col, t[p]);
            if constexpr (STREAM) {
                float r[8];
                norm_load(residual + col, r);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    t[p][i] = norm_held(residual, t[p][i] + r[i]);
                norm_store(total + col, t[p]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                squares += t[p][i] * t[p][i];
        }
    }
    const float n = 1.0f / sqrtf(norm_row_sum<THREADS>(squares, space) * a.per_width + a.eps);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const uint32_t col = (p * THREADS + lane) * 8;
        if (col < a.width && here) {
            float w[8];
            norm_load(a.weight + col, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                t[p][i] = t[p][i] * n * w[i];
            norm_store(a.y + at + col, t[p]);
        }
    }
}

// THREADS * PIECES * 8 >= width.  The workgroup's part of dw leaves to grad_weight[blockIdx.x].
template <int THREADS, int PIECES, class T>
__global__ void __launch_bounds__(kNormBackThreads) norm_back_kernel(const NormBackArgs a)
{
    constexpr uint32_t kRows = kNormBackThreads / THREADS;
    __shared__ float space[2][2][kNormBackThreads / 64];
    __shared__ float parts[kRows > 1 ? THREADS * PIECES * 8 : 8];
    const uint32_t group = threadIdx.x / THREADS, lane = threadIdx.x % THREADS;
    float w[PIECES][8], dw[PIECES][8] = {};
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const uint32_t col = (p * THREADS + lane) * 8;
        if (col < a.width)
            norm_load(a.weight + col, w[p]);
    }
    uint32_t turn = 0;
    for (uint64_t first = static_cast<uint64_t>(blockIdx.x) * kRows; first < a.tokens; first += static_cast<uint64_t>(gridDim.x) * kRows, turn ^= 1) {
        const bool here = first + group < a.tokens;
        const uint64_t at = (here ? first + group : 0) * a.width;
        const T *total = static_cast<const T *>(a.total) + at;
        float t[PIECES][8], g[PIECES][8];
        float squares = 0.0f, both = 0.0f;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const uint32_t col = (p * THREADS + lane) * 8;
            if (col < a.width && here) {
                norm_load(total + col, t[p]);
                norm_load(a.grad_y + at + col, g[p]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    squares += t[p][i] * t[p][i];
                    both += g[p][i] * w[p][i] * t[p][i];
                }
            }
        }
        squares = norm_wave_sum(squares);
        both = norm_wave_sum(both);
        if constexpr (THREADS > 64) {
            // (one barrier a turn: what this turn writes is read before the next turn's barrier, and written again behind it)
            const uint32_t wave = threadIdx.x / 64, row_first = wave / (THREADS / 64) * (THREADS / 64);
            if (threadIdx.x % 64 == 0)
                space[turn][0][wave] = squares, space[turn][1][wave] = both;
            __syncthreads();
            squares = both = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < THREADS / 64; ++i)
                squares += space[turn][0][row_first + i], both += space[turn][1][row_first + i];
        }
        const float n = 1.0f / sqrtf(squares * a.per_width + a.eps);
        const float pull = n * (both * a.per_width);  // (n^3 by itself would leave binary32 where rows are very small or large)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const uint32_t col = (p * THREADS + lane) * 8;
            if (col < a.width && here) {
                float out[8] = {};
                if (a.grad_x && a.grad_total)
                    norm_load(a.grad_total + at + col, out);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float tn = t[p][i] * n;
                    out[i] += n * (g[p][i] * w[p][i] - tn * pull);
                    dw[p][i] += g[p][i] * tn;
                }
                if (a.grad_x)
                    norm_store(a.grad_x + at + col, out);
            }
        }
    }
    if (!a.grad_weight)
        return;
    float *to = a.grad_weight + static_cast<uint64_t>(blockIdx.x) * a.width;
    // the rows' parts, one group's onto those of the groups before it
    for (uint32_t turn_of = 0; turn_of < kRows; ++turn_of) {
        if (group == turn_of) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const uint32_t col = (p * THREADS + lane) * 8;
                if (col < a.width) {
                    if (turn_of) {
                        float sum[8];
                        norm_load(parts + col, sum);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            dw[p][i] += sum[i];
                    }
                    norm_store(turn_of + 1 < kRows ? parts + col : to + col, dw[p]);
                }
            }
        }
        if (kRows > 1)
            __syncthreads();
    }
}

// dw: the sum of `count` rows of `width` floats, kNormJoinColumns columns to a workgroup, 64 runs of rows side by side.  (Its time is one way to
// memory and back: 256 rows of 4096 in 4.0 us, 84 of 1160 in 2.8.)
inline __global__ void __launch_bounds__(256) norm_join_kernel(const float *parts, float *grad_weight, uint32_t count, uint32_t width)
{
    __shared__ float4 sums[4][kNormJoinColumns / 4];
    const uint32_t x = threadIdx.x % 4, y = threadIdx.x / 4, col = blockIdx.x * kNormJoinColumns + x * 4;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (col < width)
#pragma unroll 4
        for (uint32_t r = y; r < count; r += 64) {
            const float4 v = *reinterpret_cast<const float4 *>(parts + static_cast<uint64_t>(r) * width + col);
            sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
        }
#pragma unroll
    for (int apart = 4; apart < 64; apart *= 2) {
        sum.x += __shfl_xor(sum.x, apart), sum.y += __shfl_xor(sum.y, apart);
        sum.z += __shfl_xor(sum.z, apart), sum.w += __shfl_xor(sum.w, apart);
    }
    if (threadIdx.x % 64 < 4)
        sums[threadIdx.x / 64][x] = sum;
    __syncthreads();
    if (y == 0 && col < width) {
#pragma unroll
        for (int i = 1; i < 4; ++i) {
            const float4 v = sums[i][x];
            sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
        }
        *reinterpret_cast<float4 *>(grad_weight + col) = sum;
    }
}

}  // namespace nz
