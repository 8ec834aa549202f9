// Which kernel a call of the attention takes, and into how many workgroups its work is cut.  (No device code in here: a host program can include it.)
#pragma once

#include <cstddef>
#include <cstdint>

#include "neuzip_sequences.h"

namespace nz {

constexpr uint32_t kAttendFewRows = 16, kAttendSomeRows = 32, kAttendManyRows = 128, kAttendHugeRows = 256;  // of a workgroup: a sequence's newest tokens times the query heads of a head
constexpr uint32_t kAttendStep = 64;        // keys
constexpr uint32_t kAttendCus = 256;
// That a launch is split into, where its keys allow it: two to a SIMD.  (4096: 64 sequences of 4096 tokens 99 us, with 2048 93; 48 of 2178 to 8192 113 and 108.)
constexpr uint32_t kAttendWaves = 2048;
constexpr uint32_t kAttendWaveSteps = 2;    // of each wave of a split at least, few and some rows
constexpr uint32_t kAttendManySteps = 16;   // of a split at least, many rows
constexpr uint32_t kAttendMostSplits = 128;

constexpr uint32_t attend_shift(uint32_t rows) { return rows == 16 ? 4 : rows == 32 ? 5 : rows == 128 ? 7 : 8; }

struct AttendShape {
    uint32_t rows;   // to a workgroup
    uint32_t waves;  // to a workgroup
    TileNumbers numbers;
    uint64_t tiles;
    uint32_t splits, keys, least_steps;
    uint64_t sums, bytes;  // of scratch memory: the partial sums, and with the rows' statistics
};

// Whether tiles of 128 rows, `tiles` of them with all heads, are taken rather than tiles of 32: a step costs less there and takes longer, so there
// has to be enough work for all CUs, either many tiles or, with heads of 128, few that look back far (their steps are split).  us, tiles of 32 / 128,
// 32 query heads on 8:
//   head_dim 128: prompts of 512 tokens (128 tiles of up to 8 steps) 12 / 18, 1024 (256 of 16) 28 / 31, 1280 (320) 38 / 39, 2048 (512) 68 / 60, 4 of 384
//     (384 of 6) 31 / 21, 16 of 128 (512 of 2) 34 / 16;  256 tokens behind 7936 (64 of 128) 59 / 54, 512 behind 7680 (128 of 128) 95 / 88, but 128 behind
//     8064 (32 of 128) 38 / 41 and 512 behind 3584 (128 of 64) 51 / 55
//   head_dim 64: 1024 tokens (256 of 16) 17 / 23, 2048 (512 of 32) 38 / 43, 4096 (1024) 110 / 92;  4 of 384 (384 of 6) 17 / 15, 2 of 768 (384 of 12) 21 / 20,
//     2 of 1024 (512 of 16) 28 / 29;  512 behind 7680 (128 of 128) 55 / 61
inline bool attend_is_large(uint32_t head_dim, uint64_t tiles, uint64_t steps)
{
    if (head_dim == 128)
        return tiles >= 320 || (steps >= 100 && tiles * steps >= 8192);
    return tiles >= (steps <= 12 ? 384 : 700);
}

// Whether they are tiles of 256 rows instead: keys and values are widened once for twice as many rows, but a CU has one workgroup, and nobody else's work fills its
// beginning, its end, or the time when only the last tokens' are left.  So the steps have to be many, and the tiles many or about as long as each other (few
// new tokens, `tokens` of a sequence, that look back far).  us, tiles of 128 / 256 rows, 32 query heads on 8, pages of 64: prompts of 4096 tokens 163 / 151, 8192
// 581 / 555, 2 of 4096 310 / 302, but 3000 91 / 98, 4 of 2048 172 / 173, 64 of 512 272 / 309;  1024 tokens behind 7168 160 / 147, 4 of 512 behind 3584 148 / 138,
// 512 behind 32256 299 / 275, but 2048 behind 2048 123 / 132.  In pages of 16 the prompt of 4096 takes 155 / 159.
// Several prompts: 2 of 3100 182 / 186, 2 of 3300 207 / 203, 3 of 3100 267 / 271, 3 of 4096 440 / 440, 6 of 4096 893 / 882, 3 of 6000 929 / 907, 3 of 8192 1665 / 1627; one of
// 6000 311 / 320; 4 of 1024 behind 3000 255 / 246, 8 of 300 behind 3000 195 / 200.
// (Heads of 64 have no such tiles: a step's keys are 256 pieces of 16 bytes, half as many as the threads that would ask for them.)
inline bool attend_is_largest(uint32_t head_dim, uint32_t page_tokens, uint64_t tiles, uint64_t steps, uint64_t tokens)
{
    return head_dim == 128 && page_tokens >= kAttendStep && steps >= 48 && (tiles >= 1024 || steps * kAttendStep >= 4 * tokens);
}

// heads: of the cache; count: sequences; longest: no sequence has more tokens
inline AttendShape attend_shape(uint32_t heads, uint32_t head_dim, uint32_t page_tokens, uint32_t count, uint32_t q_heads, uint32_t rows, uint32_t window, uint64_t longest)
{
    const uint32_t group = q_heads / heads;
    AttendShape shape;
    const uint64_t all = static_cast<uint64_t>(rows) * group;
    // the keys that a tile's rows see, at most
    const uint64_t span = static_cast<uint64_t>(window) + kAttendHugeRows / group + 1;
    const uint64_t keys = window && span < longest ? span : longest;
    const uint64_t large = all / kAttendManyRows * heads, steps = keys / kAttendStep;
    if (all <= static_cast<uint64_t>(count) * kAttendFewRows)
        shape.rows = kAttendFewRows;
    else if (!attend_is_large(head_dim, large, steps))
        shape.rows = kAttendSomeRows;
    else
        shape.rows = attend_is_largest(head_dim, page_tokens, large, steps, rows / count) ? kAttendHugeRows : kAttendManyRows;
    const uint32_t tile = shape.rows;
    // The fewer numbers: single tokens are counted one by one, so that none of their workgroups is empty, which would put the others unevenly
    // on the CUs (64 sequences of 4096 tokens, 32 heads on 8: 93 us, numbered in tiles 111).
    const TileNumbers in_tiles = {attend_shift(tile), group, 1}, in_rows = {0, (group + tile - 1) / tile, 0};
    shape.numbers = tile_count(in_rows, rows, count) <= tile_count(in_tiles, rows, count) ? in_rows : in_tiles;
    shape.tiles = tile_count(shape.numbers, rows, count);
    // workgroups that have something to do, about
    const uint64_t full = (all + tile - 1) / tile;
    const uint64_t wgs = (full > count ? full : count) * heads;
    // (us, 8 waves / 4: 32 sequences of 8192 tokens, 256 workgroups, 94 / 99; 48 of 5232 99 / 96, 256 of 1024 108 / 96)
    shape.waves = tile == kAttendHugeRows || (tile == kAttendFewRows && wgs <= kAttendCus) ? 8 : 4;
    shape.least_steps = tile >= kAttendManyRows ? kAttendManySteps : kAttendWaveSteps * shape.waves;
    const uint64_t wanted = (kAttendWaves + wgs * shape.waves - 1) / (wgs * shape.waves), most = keys / (kAttendStep * shape.least_steps);
    uint64_t splits = wanted < most ? wanted : most;
    splits = splits < kAttendMostSplits ? splits : kAttendMostSplits;
    shape.splits = splits ? static_cast<uint32_t>(splits) : 1;
    shape.keys = static_cast<uint32_t>(keys);
    const uint64_t parts = shape.splits > 1 ? static_cast<uint64_t>(shape.splits) * rows * q_heads : 0;
    shape.sums = (parts * head_dim * sizeof(float) + 255) / 256 * 256;
    shape.bytes = shape.sums + parts * 2 * sizeof(float);
    return shape;
}

}  // namespace nz
