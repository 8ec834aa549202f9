// Which form of the gated block's kernels a product takes: host code without a device's, which tests compile by itself.
#pragma once

#include <cstdint>

namespace nz {

enum GatedForm { kForward, kInputGrad, kWeightGrad };

constexpr uint32_t kGatedDepth = 64;  // k of a step

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
inline GatedShape gated_shape(uint64_t rows, uint64_t cols, uint64_t depth)
{
    const double steps = static_cast<double>(tiles_of(depth, kGatedDepth)) * (FORM == kInputGrad ? 2 : 1);
    // Sums of fewer than four steps fill no ring of four, and tiles of 256 are then all beginning and end: 128, two held, without a look at
    // the figures above, which are of longer sums (128 with two held / with four / 256, us: weight gradients of 8 to 192 tokens, 256 -> 640
    // 6.5-7.5 / 6.4-8.3 / 10.9-13.3, 1160 -> 2808 9.2-12.3 / 11.2-15.3 / 11.5-16.1, 4096 -> 14336 60-87 / 96-138 / 71-98; forward of 64 to 192
    // features, 64 to 2048 tokens, 4096 outputs 4.1-13.6 / 4.1-19.7 / 9.1-14.1; input gradient of 32 and 64 outputs, 4096 features,
    // 6.1-10.3 / 6.3-12.7 / 10.1-14.6.  By those figures few tiles would have four held: 7.7 -> 8.3, 4.8 -> 5.1.)
    if (steps < 4)
        return {128, 2, 1};
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
inline uint32_t gated_beside(uint64_t tokens, uint64_t out_features, uint64_t in_features)
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

}  // namespace nz
