// Which form of the linear layer's kernel a launch takes, for the layer by itself and with another's work beside it.
#pragma once

#include "neuzip_linear_kernels.h"

namespace nz {

// Workgroups up to which the walks step without a branch (see rans_get): at most one per CU, two waves per SIMD (4096 x 4096,
// 1 token, 15.5 us, with the branch 16.1; 1000 x 1024 17.0 / 17.7; 2048 x 4096, 16 tokens, k = 3, 15.5 / 16.4), while with more
// (q, k and v of a Llama-3-8B attention block, 8 tokens: 20.9 / 20.0; two of 4096 x 4096, 12 tokens: 20.8 / 19.9) the vector unit has the branch's savings.
// Not where most of the weights are symbols of 8 or of 4 bits, all alike, whose runs have 256 or 128 bytes, one as long as the
// other: the lanes of a wave then read one or two LDS banks, at every symbol without the branch (16 exponents of one frequency,
// 4096 x 4096, 1 token, 21.6 us).
constexpr uint32_t kLinEager = 256;

struct LinearLaunch {
    int k;              // mantissa bits of the weights
    bool normalised;
    bool in_step;       // most of the weights have runs of one length
    uint32_t cols, wgs;
};

template <template <int, int, int, bool, bool, bool> class Kernel, int KB, bool NORM, class... More>
void launch_linear_of(const LinearBatchArgs &batch, const LinearLaunch &kind, hipStream_t stream, const More &...more)
{
    bool read = true;  // all weights walked whole, with tables to read
    for (uint32_t i = 0; i < batch.count; ++i)
        read = read && !batch.t[i].split && holds_table(batch.t[i].n_chunks);
#define NZ_LINEAR(COLS, MT)                                                                      \
    do {                                                                                         \
        if (read)                                                                                \
            Kernel<KB, COLS, MT, NORM, true, false>::launch(batch, kind.wgs, stream, more...);   \
        else if (kind.wgs <= kLinEager && !kind.in_step)                                         \
            Kernel<KB, COLS, MT, NORM, false, true>::launch(batch, kind.wgs, stream, more...);   \
        else                                                                                     \
            Kernel<KB, COLS, MT, NORM, false, false>::launch(batch, kind.wgs, stream, more...);  \
    } while (0)
    const uint32_t tokens = batch.t[0].tokens;
    if (kind.cols == 32) {
        if (tokens <= 32)
            NZ_LINEAR(32, 1);
        else
            NZ_LINEAR(32, 2);
        return;
    }
    switch ((tokens + 15) / 16) {
    case 1: NZ_LINEAR(16, 1); break;
    case 2: NZ_LINEAR(16, 2); break;
    case 3: NZ_LINEAR(16, 3); break;
    default: NZ_LINEAR(16, 4); break;
    }
#undef NZ_LINEAR
}

// Kernel<...>::launch(batch, wgs, stream, more...) launches the form of the kernel that serves these weights and tokens.
template <template <int, int, int, bool, bool, bool> class Kernel, class... More>
void launch_linear(const LinearBatchArgs &batch, const LinearLaunch &kind, hipStream_t stream, const More &...more)
{
    if (kind.normalised) {
        switch (kind.k) {
        case 3: launch_linear_of<Kernel, 3, true>(batch, kind, stream, more...); break;
        case 1: launch_linear_of<Kernel, 1, true>(batch, kind, stream, more...); break;
        default: launch_linear_of<Kernel, 0, true>(batch, kind, stream, more...); break;
        }
    } else {
        switch (kind.k) {
        case 7: launch_linear_of<Kernel, 7, false>(batch, kind, stream, more...); break;
        case 3: launch_linear_of<Kernel, 3, false>(batch, kind, stream, more...); break;
        case 1: launch_linear_of<Kernel, 1, false>(batch, kind, stream, more...); break;
        default: launch_linear_of<Kernel, 0, false>(batch, kind, stream, more...); break;
        }
    }
}

}  // namespace nz
