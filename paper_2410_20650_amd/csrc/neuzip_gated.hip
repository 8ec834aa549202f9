// Gated feed-forward block: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "neuzip.h"

#include "neuzip_gated_kernels.h"
#include "neuzip_host.h"

using namespace nz;

namespace {

// Widths of the matrices: offsets inside a tile (256 rows) have 32 bits.
constexpr uint64_t kGatedWidest = 1ull << 22;
constexpr uint64_t kGatedMostTokens = 1ull << 31;

inline bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) & 15u; }
inline bool valid_activation(int a) { return a == NEUZIP_SILU || a == NEUZIP_GELU_TANH; }
inline bool valid_width(uint64_t w) { return w > 0 && w % 8 == 0 && w <= kGatedWidest; }

inline uint32_t tiles_of(uint64_t n, uint32_t size) { return static_cast<uint32_t>((n + size - 1) / size); }

struct GatedShape {
    uint32_t size, ring, slices;
};

// Tiles of 256 or of 128, and for the input gradient, whose tiles are few and their sums long, how many slices of k: the least of
// what the forms are expected to take, in us.  Each has a beginning, its rounds (as many tiles as the CUs have places for) of steps of 64 k, and
// what the products of all tiles take away in clock and from each other:
//   256             a step 1.0, a tile 4.3, 10^9 operations 0.2     (512 tokens, 4096 -> 14336: forward 102 us, weight gradients 141)
//   128, two to a CU    0.39, 0.5 and 0.48                          (138 and 144; 1500 tokens, 1024 -> 4096, 35.0 and 27.1, tiles of 256 36.2 and 40.6)
//   128, four steps held, no more tiles than CUs  0.35 and 0.27     (200 tokens, 4096 -> 4096, forward 29.7, two to a CU 35.7)
// and the sums of slices are written and read again in binary32 (input gradient of 2048 tokens, 4096 -> 14336: 487 us in one slice of 256, 339
// in two; of 64 tokens, 166 in one of 128, 42 in eight).  Over 19 shapes of 1 to 2048 tokens the choice takes 1.4 % more than the best one.
template <GatedForm FORM>
GatedShape gated_shape(uint64_t rows, uint64_t cols, uint64_t depth)
{
    const double steps = static_cast<double>(tiles_of(depth, kGatedDepth)) * (FORM == kInputGrad ? 2 : 1);
    GatedShape best = {128, 2, 1};
    double least = 0;
    for (uint32_t size = 128; size <= 256; size += 128) {
        const uint64_t tiles = static_cast<uint64_t>(tiles_of(rows, size)) * tiles_of(cols, FORM == kForward ? size / 2 : size) * (FORM == kWeightGrad ? 2 : 1);
        const double work = 2e-9 * size * size * kGatedDepth * steps * static_cast<double>(tiles);
        for (uint32_t slices = 1; slices <= (FORM == kInputGrad ? 16u : 1u) && steps >= 4.0 * slices; slices *= 2) {
            const uint64_t all = tiles * slices;
            const uint32_t ring = size == 128 && all <= 256 ? 4 : 2;
            const double each = steps / slices;
            double us = size == 256 ? 4 + static_cast<double>((all + 255) / 256) * (1.0 * each + 4.3) + 0.2 * work
                        : ring == 4 ? 4 + 0.35 * each + 0.27 * work
                                    : 3.3 + static_cast<double>((all + 511) / 512) * (0.39 * each + 0.5) + 0.48 * work;
            if (slices > 1)
                us += 3.0 + static_cast<double>(rows) * cols * 4 * (slices + 0.5) / 3e6;
            if (least == 0 || us < least) {
                least = us;
                best = {size, ring, slices};
            }
        }
    }
    return best;
}

// Both gradients in one launch, where both would be in tiles of 128: the input gradient's long sums run beside the weight gradients' many
// short ones.  Returns its slices, 0 for a launch each.  (333 tokens, 1160 -> 2808: 21.3 us with the join, 28.9 one behind the other; 200,
// 4096 -> 4096, 45 to 50 and 53; 1500, 1024 -> 4096, 55 and 62; a slice's step 0.65 us, a tile of the input gradient 4 more, its sums
// at 1 TB/s: over 14 shapes 2 % more than the best number of slices.)
uint32_t gated_beside(uint64_t tokens, uint64_t out_features, uint64_t in_features)
{
    if (gated_shape<kInputGrad>(tokens, in_features, out_features).size != 128 || gated_shape<kWeightGrad>(out_features, in_features, tokens).size != 128)
        return 0;
    const double x_tiles = static_cast<double>(tiles_of(tokens, 128)) * tiles_of(in_features, 128), x_steps = 2.0 * tiles_of(out_features, kGatedDepth);
    const double w_tiles = 2.0 * tiles_of(out_features, 128) * tiles_of(in_features, 128), w_steps = tiles_of(tokens, kGatedDepth);
    const double work = 2e-9 * 128 * 128 * kGatedDepth * (x_steps * x_tiles + w_steps * w_tiles);
    uint32_t best = 1;
    double least = 0;
    for (uint32_t slices = 1; slices <= 16 && x_steps >= 4.0 * slices; slices *= 2) {
        const double each = x_steps / slices;
        const double all = (x_tiles * slices * (0.39 * each + 4) + w_tiles * (0.39 * w_steps + 0.5)) / 512 + 0.48 * work;
        double us = all > 0.65 * each ? all : 0.65 * each;
        if (slices > 1)
            us += 3.0 + static_cast<double>(tokens) * in_features * 4 * (slices + 0.5) / 1e6;
        if (least == 0 || us < least) {
            least = us;
            best = slices;
        }
    }
    return best;
}

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
