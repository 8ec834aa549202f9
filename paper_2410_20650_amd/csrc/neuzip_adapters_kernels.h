// Low-rank adapters beside a projection for gfx950:  y[t] += s[a] B[a] (A[a] x[t]),  a = id[t].
//
// The low products, rank floats a token, by workgroups behind the linear layer's own in its launch, where a CU has room beside one of
// those or has run out of them; the high ones in a launch behind it: every row of A is a sum over all input features, and every output
// wants all of them.  Bound by the linear layer beside them (4096 -> 4096, one token, rank 16: 17.4 us in all, 22.0 with the low
// products in a launch in front, the layer alone 14.7; 14336 -> 4096, 48 tokens, 24 adapters of rank 64, 88 MB read by waves: 58.5, 64.1 with
// them beside the setting up of the layer's outputs).  A token reads its adapter by itself: tokens are not put in the order of their
// adapters first, which would cost a launch; those of a common one meet in the L2.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "neuzip_linear_launch.h"

namespace nz {

struct AdapterArgs {
    const uint16_t *x;      // [tokens][in_features]
    const uint16_t *a;      // [adapters][rank][in_features]
    const uint16_t *b;      // [adapters][out_features][rank]
    const float *scales;    // [adapters], or nullptr: 1
    const int32_t *ids;     // [tokens]; outside 0 .. adapters - 1: none
    float *low;             // [tokens][rank], with the scale
    float *y;               // [tokens][out_features]
    uint32_t tokens, adapters, rank, in_features, out_features;
};

__device__ __forceinline__ float adapter_low_half(uint32_t d) { return __uint_as_float(d << 16); }
__device__ __forceinline__ float adapter_high_half(uint32_t d) { return __uint_as_float(d & 0xFFFF0000u); }
__device__ __forceinline__ float adapter_dot(const uint4 &p, const uint4 &q, float sum)
{
    const uint32_t ps[4] = {p.x, p.y, p.z, p.w}, qs[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum = fmaf(adapter_low_half(ps[i]), adapter_low_half(qs[i]), sum);
        sum = fmaf(adapter_high_half(ps[i]), adapter_high_half(qs[i]), sum);
    }
    return sum;
}

// low[t][r] = s (A[a] x[t])[r]: a wave to a token and a row of A.
constexpr uint32_t kAdapterRows = kLinThreads / 64;  // rows of A of a workgroup
__device__ __forceinline__ void adapter_low_workgroup(const AdapterArgs &g, uint32_t wg)
{
    const uint32_t groups = (g.rank + kAdapterRows - 1) / kAdapterRows, t = wg / groups;
    const uint32_t lane = threadIdx.x % 64, r = (wg - t * groups) * kAdapterRows + threadIdx.x / 64;
    const int32_t id = g.ids[t];
    if (r >= g.rank || id < 0 || static_cast<uint32_t>(id) >= g.adapters)
        return;
    const uint4 *x = reinterpret_cast<const uint4 *>(g.x + static_cast<uint64_t>(t) * g.in_features);
    const uint4 *a = reinterpret_cast<const uint4 *>(g.a + (static_cast<uint64_t>(id) * g.rank + r) * g.in_features);
    // (eight pieces of both requested together; in_features is a multiple of 128, so lanes end apart)
    const uint32_t pieces = g.in_features / 8;
    float sum = 0.0f;
    for (uint32_t i0 = lane; i0 < pieces; i0 += 64 * 8) {
        uint4 xs[8], as[8];
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k) {
            const uint32_t i = min(i0 + k * 64, pieces - 1);
            xs[k] = x[i];
            as[k] = a[i];
        }
#pragma unroll
        for (uint32_t k = 0; k < 8; ++k)
            if (i0 + k * 64 < pieces)
                sum = adapter_dot(xs[k], as[k], sum);
    }
#pragma unroll
    for (int apart = 32; apart > 0; apart /= 2)
        sum += __shfl_xor(sum, apart);
    if (lane == 0)
        g.low[static_cast<uint64_t>(t) * g.rank + r] = g.scales ? g.scales[id] * sum : sum;
}

// The linear layer's workgroups, and behind them those of the low products.
template <int KB, int COLS, int MT, bool NORM, bool READ, bool EAGER>
__global__ __launch_bounds__(kLinThreads, 4) void linear_adapters_kernel(const LinearBatchArgs b, const AdapterArgs g, const uint32_t wgs)
{
    if (blockIdx.x < wgs)
        linear_batch_workgroup<KB, COLS, MT, NORM, READ, EAGER>(b);
    else
        adapter_low_workgroup(g, blockIdx.x - wgs);
}

// y[t][o] += B[a][o] . low[t]: a thread to an output.
constexpr uint32_t kAdapterThreads = 256;
__global__ __launch_bounds__(kAdapterThreads) void adapter_high_kernel(const AdapterArgs g)
{
    const uint32_t o = blockIdx.x * kAdapterThreads + threadIdx.x, t = blockIdx.y;
    const int32_t id = g.ids[t];
    if (o >= g.out_features || id < 0 || static_cast<uint32_t>(id) >= g.adapters)
        return;
    const uint4 *b = reinterpret_cast<const uint4 *>(g.b + (static_cast<uint64_t>(id) * g.out_features + o) * g.rank);
    const float *low = g.low + static_cast<uint64_t>(t) * g.rank;
    float sum = 0.0f;
#pragma unroll 4
    for (uint32_t i = 0; i < g.rank / 8; ++i) {
        const uint4 v = b[i];
        const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            sum = fmaf(adapter_low_half(d[p]), low[8 * i + 2 * p], sum);
            sum = fmaf(adapter_high_half(d[p]), low[8 * i + 2 * p + 1], sum);
        }
    }
    g.y[static_cast<uint64_t>(t) * g.out_features + o] += sum;
}

}  // namespace nz
