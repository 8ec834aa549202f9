// Root-mean-square norm with the residual's addition: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cstdint>

#include "neuzip.h"

#include "neuzip_host.h"
#include "neuzip_norm_kernels.h"

using namespace nz;

namespace {

constexpr uint64_t kNormWidest = 16384;
constexpr uint64_t kNormMostTokens = 1ull << 24;

inline bool misaligned(const void *p) { return reinterpret_cast<uintptr_t>(p) & 15u; }
inline bool valid_type(int t) { return t == NEUZIP_F32 || t == NEUZIP_BF16; }
inline bool valid_width(uint64_t w) { return w > 0 && w % 8 == 0 && w <= kNormWidest; }
inline bool valid_eps(float eps) { return eps >= 0.0f; }  // (no NaN)

// A launch has fewer than 2^32 threads: with 1024 to a row, 2^22 tokens and more are several.
template <int THREADS, int PIECES, class X, bool STREAM, class T>
void launch_norm_as(const NormArgs &a, hipStream_t stream)
{
    constexpr uint32_t threads = THREADS > static_cast<int>(kNormThreads) ? THREADS : kNormThreads, rows = threads / THREADS;
    constexpr uint32_t most = ((1ull << 32) / threads - 1) * rows;
    static_assert(too_many_wgs(most / rows + 1, threads) && !too_many_wgs(most / rows, threads) && (threads > kNormThreads || most >= kNormMostTokens - 1));
    for (uint32_t first = 0; first < a.tokens; first += most) {
        const uint64_t at = static_cast<uint64_t>(first) * a.width;
        NormArgs part = a;
        part.x = static_cast<const X *>(a.x) + at;
        part.y = a.y + at;
        if constexpr (STREAM) {
            part.residual = static_cast<const T *>(a.residual) + at;
            part.total = static_cast<T *>(a.total) + at;
        }
        part.tokens = a.tokens - first < most ? a.tokens - first : most;
        hipLaunchKernelGGL((norm_kernel<THREADS, PIECES, X, STREAM, T>), dim3((part.tokens + rows - 1) / rows), dim3(threads), 0, stream, part);
    }
}

// us, a wave / 256 lanes to a row: 4096 rows of 512 4.4 / 5.5, 32768 of them 26.6 / 34.5; 333 rows of 1024 2.8 / 2.5 and 4096 of them 7.1 / 7.9.
template <class X, bool STREAM, class T>
void launch_norm(const NormArgs &a, hipStream_t stream)
{
    if (a.width <= 512)
        launch_norm_as<64, 1, X, STREAM, T>(a, stream);
    else if (a.width <= 2048)
        launch_norm_as<256, 1, X, STREAM, T>(a, stream);
    else if (a.width <= 4096)
        launch_norm_as<256, 2, X, STREAM, T>(a, stream);
    else if (a.width <= 8192)
        launch_norm_as<256, 4, X, STREAM, T>(a, stream);
    else
        launch_norm_as<1024, 2, X, STREAM, T>(a, stream);
}

template <class X>
void launch_norm_of(const NormArgs &a, int total_type, hipStream_t stream)
{
    if (!a.total)
        launch_norm<X, false, X>(a, stream);
    else if (total_type == NEUZIP_F32)
        launch_norm<X, true, float>(a, stream);
    else
        launch_norm<X, true, uint16_t>(a, stream);
}

// Lanes to a row of the backward pass.
inline uint32_t back_threads(uint64_t width) { return width <= 1024 ? 64 : width <= 4096 ? 256 : 1024; }

inline uint32_t back_wgs(uint64_t tokens, uint64_t width)
{
    const uint64_t rows = kNormBackThreads / back_threads(width), wgs = (tokens + rows - 1) / rows;
    return static_cast<uint32_t>(wgs < kNormMostWgs ? wgs : kNormMostWgs);
}

template <int THREADS, int PIECES, class T>
void launch_back_as(const NormBackArgs &a, uint32_t wgs, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_back_kernel<THREADS, PIECES, T>), dim3(wgs), dim3(kNormBackThreads), 0, stream, a);
}

template <class T>
void launch_back(const NormBackArgs &a, uint32_t wgs, hipStream_t stream)
{
    if (a.width <= 512)
        launch_back_as<64, 1, T>(a, wgs, stream);
    else if (a.width <= 1024)
        launch_back_as<64, 2, T>(a, wgs, stream);
    else if (a.width <= 2048)
        launch_back_as<256, 1, T>(a, wgs, stream);
    else if (a.width <= 4096)
        launch_back_as<256, 2, T>(a, wgs, stream);
    else if (a.width <= 8192)
        launch_back_as<1024, 1, T>(a, wgs, stream);
    else
        launch_back_as<1024, 2, T>(a, wgs, stream);
}

}  // namespace

extern "C" {

int neuzip_norm(const void *d_x, int x_type, const void *d_residual, void *d_total, int total_type, const float *d_weight, uint64_t tokens,
                uint64_t width, float eps, void *d_y, void *hip_stream)
{
    if (!valid_type(x_type) || !valid_type(total_type) || !valid_width(width) || !valid_eps(eps) || !d_residual != !d_total ||
        (!d_total && total_type != x_type))
        return NEUZIP_EINVAL;
    if (tokens == 0)
        return NEUZIP_OK;
    if (!d_x || !d_weight || !d_y)
        return NEUZIP_EINVAL;
    const void *const pointers[] = {d_x, d_residual, d_total, d_weight, d_y};
    for (const void *p : pointers)
        if (misaligned(p))
            return NEUZIP_EINVAL;
    if (tokens >= kNormMostTokens)
        return NEUZIP_EUNSUPPORTED;
    NormArgs a;
    a.x = d_x;
    a.residual = d_residual;
    a.total = d_total;
    a.weight = d_weight;
    a.y = static_cast<uint16_t *>(d_y);
    a.tokens = static_cast<uint32_t>(tokens);
    a.width = static_cast<uint32_t>(width);
    a.eps = eps;
    a.per_width = 1.0f / static_cast<float>(width);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (x_type == NEUZIP_F32)
        launch_norm_of<float>(a, total_type, stream);
    else
        launch_norm_of<uint16_t>(a, total_type, stream);
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

uint64_t neuzip_norm_backward_scratch_bytes(uint64_t tokens, uint64_t width)
{
    if (!valid_width(width) || tokens >= kNormMostTokens)
        return 0;
    // (one workgroup's part is the whole)
    const uint32_t wgs = back_wgs(tokens, width);
    return wgs > 1 ? wgs * width * sizeof(float) : 0;
}

int neuzip_norm_backward(const void *d_total, int total_type, const float *d_weight, const void *d_grad_y, const void *d_grad_total,
                         uint64_t tokens, uint64_t width, float eps, void *d_grad_x, float *d_grad_weight, void *d_scratch,
                         uint64_t scratch_bytes, void *hip_stream)
{
    if (!valid_type(total_type) || !valid_width(width) || !valid_eps(eps))
        return NEUZIP_EINVAL;
    if (tokens >= kNormMostTokens)
        return NEUZIP_EUNSUPPORTED;
    if ((tokens > 0 && (!d_total || !d_grad_y || !d_weight)) || (tokens == 0 && d_grad_weight && !d_weight))
        return NEUZIP_EINVAL;
    const void *const pointers[] = {d_total, d_weight, d_grad_y, d_grad_total, d_grad_x, d_grad_weight, d_scratch};
    for (const void *p : pointers)
        if (misaligned(p))
            return NEUZIP_EINVAL;
    const uint64_t room = neuzip_norm_backward_scratch_bytes(tokens, width);
    if (d_grad_weight && room && (!d_scratch || scratch_bytes < room))
        return NEUZIP_EINVAL;
    if (!d_grad_weight && (!d_grad_x || tokens == 0))
        return NEUZIP_OK;
    const uint32_t wgs = tokens ? back_wgs(tokens, width) : 1;  // (no tokens: one that has nothing to add)
    NormBackArgs a;
    a.total = d_total;
    a.weight = d_weight;
    a.grad_y = static_cast<const uint16_t *>(d_grad_y);
    a.grad_total = static_cast<const uint16_t *>(d_grad_total);
    a.grad_x = static_cast<uint16_t *>(d_grad_x);
    a.grad_weight = !d_grad_weight ? nullptr : room ? static_cast<float *>(d_scratch) : d_grad_weight;
    a.tokens = static_cast<uint32_t>(tokens);
    a.width = static_cast<uint32_t>(width);
    a.eps = eps;
    a.per_width = 1.0f / static_cast<float>(width);
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (total_type == NEUZIP_F32)
        launch_back<float>(a, wgs, stream);
    else
        launch_back<uint16_t>(a, wgs, stream);
    if (!hip_ok(hipGetLastError()))
        return NEUZIP_EHIP;
    if (d_grad_weight && room) {
        hipLaunchKernelGGL(norm_join_kernel, dim3((a.width + kNormJoinColumns - 1) / kNormJoinColumns), dim3(256), 0, stream,
                           static_cast<const float *>(d_scratch), d_grad_weight, wgs, a.width);
        if (!hip_ok(hipGetLastError()))
            return NEUZIP_EHIP;
    }
    return NEUZIP_OK;
}

}  // extern "C"
