// Gated feed-forward block: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "neuzip.h"

#include "neuzip_gated_kernels.h"
#include "neuzip_gated_shape.h"
#include "neuzip_host.h"

using namespace nz;

namespace {

// Widths of the matrices: offsets inside a tile (256 rows) have 32 bits.
constexpr uint64_t kGatedWidest = 1ull << 22;
constexpr uint64_t kGatedMostTokens = 1ull << 31;

inline bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) & 15u; }
inline bool valid_activation(int a) { return a == NEUZIP_SILU || a == NEUZIP_GELU_TANH; }
inline bool valid_width(uint64_t w) { return w > 0 && w % 8 == 0 && w <= kGatedWidest; }

// The tiles' numbers; returns how many workgroups compute them.
template <GatedForm FORM>
uint64_t set_tiles(GatedArgs &a, uint32_t size, uint32_t slices)
{
    a.tiles_i = tiles_of(a.rows, size);
    a.tiles_j = tiles_of(a.cols, FORM == kForward ? size / 2 : size);
    a.slices = slices;
    return static_cast<uint64_t>(a.tiles_i) * a.tiles_j * slices * (FORM == kWeightGrad ? 2 : 1);
}

template <GatedForm FORM>
int launch_gated(GatedArgs &a, const GatedShape &shape, hipStream_t stream)
{
    const uint64_t grid = set_tiles<FORM>(a, shape.size, shape.slices);
    if (too_many_wgs(grid, kGatedThreads))
        return NEUZIP_EUNSUPPORTED;
    const dim3 wgs(static_cast<uint32_t>(grid)), threads(kGatedThreads);
    if (shape.size == 256)
        hipLaunchKernelGGL((gated_kernel<FORM, 256, 2>), wgs, threads, 0, stream, a);
    else if (shape.ring == 4)
        hipLaunchKernelGGL((gated_kernel<FORM, 128, 4>), wgs, threads, 0, stream, a);
    else
        hipLaunchKernelGGL((gated_kernel<FORM, 128, 2>), wgs, threads, 0, stream, a);
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

inline uint64_t wgs_for(uint64_t threads) { return (threads + kGatedSlopeThreads - 1) / kGatedSlopeThreads; }

}  // namespace

extern "C" {

int neuzip_gated_forward(const void *d_x, const void *d_gate_weight, const void *d_up_weight, uint64_t tokens,
                         uint64_t out_features, uint64_t in_features, int activation, void *d_h, float *d_gate, float *d_up,
                         void *hip_stream)
{
    if (!valid_activation(activation) || !valid_width(out_features) || !valid_width(in_features) || tokens >= kGatedMostTokens)
        return NEUZIP_EINVAL;
    if (tokens == 0)
        return NEUZIP_OK;
    if (!d_x || !d_gate_weight || !d_up_weight || !d_h || !d_gate != !d_up)
        return NEUZIP_EINVAL;
    const void *const pointers[] = {d_x, d_gate_weight, d_up_weight, d_h, d_gate, d_up};
    for (const void *p : pointers)
        if (misaligned(p))
            return NEUZIP_EINVAL;
    GatedArgs a;
    std::memset(&a, 0, sizeof(a));
    a.q[0] = a.q[1] = static_cast<const uint16_t *>(d_x);
    a.p[0] = static_cast<const uint16_t *>(d_gate_weight);
    a.p[1] = static_cast<const uint16_t *>(d_up_weight);
    a.c[0] = static_cast<uint16_t *>(d_h);
    a.gate = d_gate;
    a.up = d_up;
    a.rows = static_cast<uint32_t>(tokens);
    a.cols = a.c_row = static_cast<uint32_t>(out_features);
    a.depth = a.q_row = a.p_row = static_cast<uint32_t>(in_features);
    a.activation = static_cast<uint32_t>(activation);
    return launch_gated<kForward>(a, gated_shape<kForward>(a.rows, a.cols, a.depth), static_cast<hipStream_t>(hip_stream));
}

uint64_t neuzip_gated_backward_scratch_bytes(uint64_t tokens, uint64_t out_features, uint64_t in_features)
{
    if (!valid_width(out_features) || !valid_width(in_features) || tokens == 0 || tokens >= kGatedMostTokens)
        return 0;
    const uint32_t alone = gated_shape<kInputGrad>(tokens, in_features, out_features).slices, beside = gated_beside(tokens, out_features, in_features);
    const uint32_t slices = alone > beside ? alone : beside;
    return 2 * pad_to(tokens * out_features * 2, 256) + (slices > 1 ? slices * tokens * in_features * sizeof(float) : 0);
}

int neuzip_gated_backward(const void *d_x, const void *d_gate_weight, const void *d_up_weight, const float *d_gate, const float *d_up,
                          const void *d_grad_h, uint64_t tokens, uint64_t out_features, uint64_t in_features, int activation,
                          void *d_grad_x, void *d_grad_gate_weight, void *d_grad_up_weight, void *d_scratch, uint64_t scratch_bytes,
                          void *hip_stream)
{
    if (!valid_activation(activation) || !valid_width(out_features) || !valid_width(in_features) || tokens >= kGatedMostTokens)
        return NEUZIP_EINVAL;
    if (!d_grad_gate_weight != !d_grad_up_weight)
        return NEUZIP_EINVAL;
    const bool weights = d_grad_gate_weight != nullptr;
    if (tokens > 0 && (!d_gate || !d_up || !d_grad_h || !d_scratch || (weights && !d_x) || (d_grad_x && (!d_gate_weight || !d_up_weight)) ||
                       scratch_bytes < neuzip_gated_backward_scratch_bytes(tokens, out_features, in_features)))
        return NEUZIP_EINVAL;
    const void *const pointers[] = {d_x, d_gate_weight, d_up_weight, d_gate, d_up, d_grad_h, d_grad_x, d_grad_gate_weight, d_grad_up_weight, d_scratch};
    for (const void *p : pointers)
        if (misaligned(p))
            return NEUZIP_EINVAL;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    uint16_t *dg = static_cast<uint16_t *>(d_scratch);
    uint16_t *du = dg + pad_to(tokens * out_features * 2, 256) / 2;
    float *partial = reinterpret_cast<float *>(du + pad_to(tokens * out_features * 2, 256) / 2);
    if (too_many_wgs(wgs_for(tokens * out_features / 8), kGatedSlopeThreads) || too_many_wgs(wgs_for(tokens * in_features / 8), kGatedSlopeThreads))
        return NEUZIP_EUNSUPPORTED;
    if (tokens > 0) {
        const uint64_t pieces = tokens * out_features / 8;
        hipLaunchKernelGGL(gated_slope_kernel, dim3(static_cast<uint32_t>(wgs_for(pieces))), dim3(kGatedSlopeThreads), 0, stream,
                           reinterpret_cast<const float4 *>(d_gate), reinterpret_cast<const float4 *>(d_up), static_cast<const uint4 *>(d_grad_h),
                           reinterpret_cast<uint4 *>(dg), reinterpret_cast<uint4 *>(du), pieces, static_cast<uint32_t>(activation));
        if (!hip_ok(hipGetLastError()))
            return NEUZIP_EHIP;
    }
    GatedArgs x, w;
    std::memset(&x, 0, sizeof(x));
    std::memset(&w, 0, sizeof(w));
    x.q[0] = w.q[0] = dg;
    x.q[1] = w.q[1] = du;
    x.p[0] = static_cast<const uint16_t *>(d_gate_weight);
    x.p[1] = static_cast<const uint16_t *>(d_up_weight);
    x.c[0] = static_cast<uint16_t *>(d_grad_x);
    x.rows = static_cast<uint32_t>(tokens);
    x.cols = x.c_row = x.p_row = static_cast<uint32_t>(in_features);
    x.depth = x.q_row = static_cast<uint32_t>(out_features);
    w.p[0] = w.p[1] = static_cast<const uint16_t *>(d_x);
    w.c[0] = static_cast<uint16_t *>(d_grad_gate_weight);
    w.c[1] = static_cast<uint16_t *>(d_grad_up_weight);
    w.rows = w.q_row = static_cast<uint32_t>(out_features);
    w.cols = w.c_row = w.p_row = static_cast<uint32_t>(in_features);
    w.depth = static_cast<uint32_t>(tokens);
    const bool input = d_grad_x && tokens > 0;
    const uint32_t beside = input && weights ? gated_beside(tokens, out_features, in_features) : 0;
    if (input) {
        GatedShape shape = gated_shape<kInputGrad>(x.rows, x.cols, x.depth);
        if (beside)
            shape.slices = beside;
        x.partial = shape.slices > 1 ? partial : nullptr;
        if (beside) {
            const uint64_t x_wgs = set_tiles<kInputGrad>(x, 128, beside), w_wgs = set_tiles<kWeightGrad>(w, 128, 1);
            if (too_many_wgs(x_wgs + w_wgs, kGatedThreads))
                return NEUZIP_EUNSUPPORTED;
            hipLaunchKernelGGL(gated_gradients_kernel, dim3(static_cast<uint32_t>(x_wgs + w_wgs)), dim3(kGatedThreads), 0, stream, x, w,
                               static_cast<uint32_t>(x_wgs));
            if (!hip_ok(hipGetLastError()))
                return NEUZIP_EHIP;
        } else {
            const int rc = launch_gated<kInputGrad>(x, shape, stream);
            if (rc != NEUZIP_OK)
                return rc;
        }
        if (shape.slices > 1) {
            const uint64_t pieces = tokens * in_features / 8;
            hipLaunchKernelGGL(gated_join_kernel, dim3(static_cast<uint32_t>(wgs_for(pieces))), dim3(kGatedSlopeThreads), 0, stream,
                               reinterpret_cast<const float4 *>(partial), static_cast<uint4 *>(d_grad_x), pieces, shape.slices);
            if (!hip_ok(hipGetLastError()))
                return NEUZIP_EHIP;
        }
    }
    if (weights && !beside)
        return launch_gated<kWeightGrad>(w, gated_shape<kWeightGrad>(w.rows, w.cols, w.depth), stream);
    return NEUZIP_OK;
}

uint64_t neuzip_gated_linear_scratch_bytes(uint64_t out_features, uint64_t in_features, uint32_t tokens)
{
    const uint64_t outs[2] = {out_features, out_features};
    return 2 * pad_to(static_cast<uint64_t>(tokens) * out_features * sizeof(float), 256) +
           neuzip_linear_scratch_bytes(outs, 2, in_features, tokens);
}

int neuzip_gated_linear(const neuzip_blob *gate, const neuzip_blob *up, uint64_t out_features, uint64_t in_features, const void *d_x,
                        uint32_t tokens, int activation, void *d_h, void *d_scratch, uint64_t scratch_bytes, void *hip_stream)
{
    if (!valid_activation(activation) || !d_h || !d_scratch || misaligned(d_scratch) || (reinterpret_cast<uintptr_t>(d_h) & 1u) ||
        tokens == 0 || out_features == 0 || out_features >= (1ull << 31) ||
        scratch_bytes < neuzip_gated_linear_scratch_bytes(out_features, in_features, tokens))
        return NEUZIP_EINVAL;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const uint64_t count = tokens * out_features, each = pad_to(count * sizeof(float), 256);
    const uint64_t wgs = wgs_for((count + 3) / 4);
    if (too_many_wgs(wgs, kGatedSlopeThreads))
        return NEUZIP_EUNSUPPORTED;
    float *const sums[2] = {static_cast<float *>(d_scratch), static_cast<float *>(d_scratch) + each / sizeof(float)};
    const neuzip_blob *const weights[2] = {gate, up};
    const uint64_t outs[2] = {out_features, out_features};
    const int rc = neuzip_linear_batch_scratch(weights, outs, 2, in_features, d_x, tokens, nullptr, sums, sums[1] + each / sizeof(float),
                                               scratch_bytes - 2 * each, hip_stream);
    if (rc != NEUZIP_OK)
        return rc;
    hipLaunchKernelGGL(gated_product_kernel, dim3(static_cast<uint32_t>(wgs)), dim3(kGatedSlopeThreads), 0, stream, sums[0],
                       sums[1], static_cast<uint16_t *>(d_h), count, static_cast<uint32_t>(activation));
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

}  // extern "C"
