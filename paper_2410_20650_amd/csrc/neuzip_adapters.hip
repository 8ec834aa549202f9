// Low-rank adapters beside a compressed projection: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "neuzip.h"

#include "neuzip_adapters_kernels.h"
#include "neuzip_host.h"

using namespace nz;

namespace {

constexpr uint32_t kAdapterMostRank = 512;
constexpr uint32_t kAdapterMostTokens = 65535;  // a grid's second dimension

inline uint64_t low_bytes(uint32_t tokens, uint32_t rank) { return pad_to(static_cast<uint64_t>(tokens) * rank * sizeof(float), 256); }

inline uint64_t low_wgs(const AdapterArgs &g) { return static_cast<uint64_t>((g.rank + kAdapterRows - 1) / kAdapterRows) * g.tokens; }

template <int KB, int COLS, int MT, bool NORM, bool READ, bool EAGER>
struct LinearAdapters {
    static void launch(const LinearBatchArgs &batch, uint32_t wgs, hipStream_t stream, const AdapterArgs &g)
    {
        hipLaunchKernelGGL((linear_adapters_kernel<KB, COLS, MT, NORM, READ, EAGER>), dim3(wgs + static_cast<uint32_t>(low_wgs(g))), dim3(kLinThreads),
                           0, stream, batch, g, wgs);
    }
};

int launch_adapters(const LinearBatchArgs &batch, const LinearLaunch &kind, const void *context, hipStream_t stream)
{
    const AdapterArgs &g = *static_cast<const AdapterArgs *>(context);
    if (too_many_wgs(kind.wgs + low_wgs(g), kLinThreads))
        return NEUZIP_EUNSUPPORTED;
    launch_linear<LinearAdapters>(batch, kind, stream, g);
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

}  // namespace

extern "C" {

uint64_t neuzip_linear_adapters_scratch_bytes(uint64_t out_features, uint64_t in_features, uint32_t tokens, uint32_t rank)
{
    return low_bytes(tokens, rank) + neuzip_linear_scratch_bytes(&out_features, 1, in_features, tokens);
}

int neuzip_linear_adapters(const neuzip_blob *weight, uint64_t out_features, uint64_t in_features, const void *d_x, uint32_t tokens,
                           const float *d_bias, const void *d_a, const void *d_b, uint32_t rank, uint32_t adapters,
                           const float *d_scales, const int32_t *d_ids, float *d_y, void *d_scratch, uint64_t scratch_bytes,
                           void *hip_stream)
{
    if (!d_a || !d_b || !d_ids || !d_scratch || rank == 0 || rank % 8 != 0 || rank > kAdapterMostRank || adapters == 0 ||
        adapters >= (1u << 31))
        return NEUZIP_EINVAL;
    if ((reinterpret_cast<uintptr_t>(d_a) & 15u) || (reinterpret_cast<uintptr_t>(d_b) & 15u) || (reinterpret_cast<uintptr_t>(d_scratch) & 15u) ||
        (reinterpret_cast<uintptr_t>(d_scales) & 3u) || (reinterpret_cast<uintptr_t>(d_ids) & 3u))
        return NEUZIP_EINVAL;
    if (tokens > kAdapterMostTokens)
        return NEUZIP_EUNSUPPORTED;
    if (scratch_bytes < neuzip_linear_adapters_scratch_bytes(out_features, in_features, tokens, rank))
        return NEUZIP_EINVAL;
    const uint64_t own = low_bytes(tokens, rank);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    AdapterArgs g;
    std::memset(&g, 0, sizeof(g));
    g.x = static_cast<const uint16_t *>(d_x);
    g.a = static_cast<const uint16_t *>(d_a);
    g.b = static_cast<const uint16_t *>(d_b);
    g.scales = d_scales;
    g.ids = d_ids;
    g.low = static_cast<float *>(d_scratch);
    g.y = d_y;
    g.tokens = tokens;
    g.adapters = adapters;
    g.rank = rank;
    g.in_features = static_cast<uint32_t>(in_features);
    g.out_features = static_cast<uint32_t>(out_features);
    const int rc = linear_with(&weight, &out_features, 1, in_features, d_x, tokens, &d_bias, &d_y, static_cast<uint8_t *>(d_scratch) + own,
                               scratch_bytes - own, launch_adapters, &g, stream);
    if (rc != NEUZIP_OK)
        return rc;
    hipLaunchKernelGGL(adapter_high_kernel, dim3((g.out_features + kAdapterThreads - 1) / kAdapterThreads, tokens), dim3(kAdapterThreads), 0,
                       stream, g);
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

}  // extern "C"
