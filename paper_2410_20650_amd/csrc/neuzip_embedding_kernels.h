// Embedding on a compressed table for gfx950: rows decoded by token, and the table's gradient.
#pragma once

#include "neuzip_format.h"
#include "neuzip_walk.h"

namespace nz {

// ------------------------------------------------------------------------------------------
// Lookup:  out[t] = bf16(scale * W_hat[token[t]]).
//
// A row lies in one chunk or in neighbouring ones, somewhere in it, and a state is decoded from its beginning or its entry point
// on.  So the unit of work is a row's share of one chunk (of half a chunk, where the blob has entry points): 16 lanes walk the
// chunk's 16 states up to the last turn that the row needs and leave the turns that belong to it, 16 bytes per lane and turn.  A wave takes four units.  Each copies its chunk's
// words straight into its wave's window of LDS, beside the slot table that the workgroup's waves share.
// ------------------------------------------------------------------------------------------
struct EmbeddingArgs {
    const TableBlock *tb;
    const uint32_t *offsets;
    const uint32_t *states;
    const uint8_t *lens;
    const uint32_t *mid_states;  // entry points (nullptr: none)
    const uint8_t *mid_lens;
    const uint16_t *words;
    const uint8_t *sm;
    const uint8_t *coef;
    uint32_t block_shift;
    uint32_t n_chunks;
    uint32_t *status;
    const int64_t *tokens;
    uint16_t *out;
    uint32_t rows, features;
    Divisor per_token;   // units of a token
    uint32_t units;
    float scale;
};

constexpr uint32_t kEmbWindow = 7680;  // bytes of LDS for the words of a wave's four chunks
constexpr uint32_t kEmbAhead = 4;      // turns whose fields are requested together

template <int KB, bool LONE, bool NORM, bool EAGER, class WordSrc>
__device__ __forceinline__ void embedding_walk(const uint32_t *__restrict__ lut, const WordSrc &src, uint32_t lone, uint32_t &x,
                                               uint32_t &wp, const EmbeddingArgs &a, uint32_t from, uint32_t lo, uint32_t hi,
                                               uint32_t turns, uint32_t most_turns, uint16_t *__restrict__ out)
{
    // this lane's runs begin at from, from + 128, ...; those inside lo .. hi - 1 belong to the row, which begins at out
    uint32_t next = LONE ? 0u : src.peek(wp);
    auto request = [&](uint32_t q) {
        const uint32_t at = from + q * kTurn;
        const uint32_t here = at < lo ? lo : (at < hi ? at : hi - kRun);  // (some run of the row)
        uint64_t f = load_fields<KB>(a.sm, here);
        if constexpr (NORM)
            f |= static_cast<uint64_t>(a.coef[here >> a.block_shift]) << 32;
        return f;
    };
    uint64_t fields[kEmbAhead] = {};
    if (turns > 0)
#pragma unroll
        for (uint32_t r = 0; r < kEmbAhead; ++r)
            fields[r] = request(r);
    for (uint32_t q0 = 0; q0 < most_turns; q0 += kEmbAhead) {
        uint64_t ahead[kEmbAhead] = {};
        if (q0 + kEmbAhead < turns)
#pragma unroll
            for (uint32_t r = 0; r < kEmbAhead; ++r)
                ahead[r] = request(q0 + kEmbAhead + r);
#pragma unroll
        for (uint32_t r = 0; r < kEmbAhead; ++r) {
            const uint32_t at = from + (q0 + r) * kTurn;
            if (q0 + r < turns && at < hi) {
                uint32_t e[8];
#pragma unroll
                for (int t = 0; t < 8; ++t)
                    e[t] = LONE ? lone : rans_get<EAGER>(lut, x, wp, next, src);
                if (at >= lo) {
                    uint32_t d[4] = {merge_pair<KB>(fields[r], 0, e[0], e[1]), merge_pair<KB>(fields[r], 1, e[2], e[3]),
                                     merge_pair<KB>(fields[r], 2, e[4], e[5]), merge_pair<KB>(fields[r], 3, e[6], e[7])};
                    if constexpr (NORM) {
                        const float c = coefficient(static_cast<uint32_t>(fields[r] >> 32) & 0x7Fu);
#pragma unroll
                        for (int p = 0; p < 4; ++p)
                            d[p] = denormalise_pair(d[p], c);
                    }
                    if (a.scale != 1.0f) {  // (unscaled, every word stays as it is, whatever it holds)
#pragma unroll
                        for (int p = 0; p < 4; ++p)
                            d[p] = bf16_of(__fmul_rn(__uint_as_float(d[p] << 16), a.scale)) |
                                   (bf16_of(__fmul_rn(__uint_as_float(d[p] & 0xFFFF0000u), a.scale)) << 16);
                    }
                    *reinterpret_cast<uint4 *>(out + (at - lo)) = make_uint4(d[0], d[1], d[2], d[3]);
                }
            }
            fields[r] = ahead[r];
        }
    }
}

template <int KB, bool NORM, bool EAGER, int THREADS>
__global__ __launch_bounds__(THREADS) void embedding_kernel(const EmbeddingArgs a)
{
    constexpr uint32_t kWaves = THREADS / 64;
    __shared__ __align__(16) struct {
        uint8_t stage[kWaves * kEmbWindow];  // first: a direct copy's LDS address has 16 bits
        uint32_t lut[kM];
        uint32_t steps[kSteps];
    } lds;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, j = tid & (kStates - 1);
    const uint32_t wave = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(tid >> 6)));
    const bool split = a.mid_states != nullptr;
    const uint32_t granule_shift = split ? 11u : 12u;
    static_assert(kChunk == 1u << 12 && kMidTurn * kTurn == 1u << 11, "log2 of a unit's elements");

    // ---- which share of which row
    const uint32_t unit = blockIdx.x * (THREADS / kStates) + tid / kStates;
    const uint32_t t = unit < a.units ? a.per_token.quotient(unit) : 0u, part = unit - t * a.per_token.by;
    const int64_t token = unit < a.units ? a.tokens[t] : -1;
    const bool valid = token >= 0 && token < static_cast<int64_t>(a.rows);
    const uint32_t row0 = valid ? static_cast<uint32_t>(token) * a.features : 0u, row1 = row0 + a.features;
    const uint32_t granule = (row0 >> granule_shift) + part;
    const uint64_t first = static_cast<uint64_t>(granule) << granule_shift;  // its first element
    const bool live = valid && first < row1;
    const uint32_t begin = live ? static_cast<uint32_t>(first) : 0u;
    const uint32_t lo = live ? max(row0, begin) : 0u;
    const uint32_t hi = live ? static_cast<uint32_t>(min(static_cast<uint64_t>(row1), first + (1ull << granule_shift))) : kRun;
    const uint32_t turns = live ? (hi - begin + kTurn - 1) / kTurn : 0u;
    const uint32_t c = begin / kChunk, behind = split && live ? granule & 1u : 0u;
    uint16_t *out = a.out + static_cast<uint64_t>(t) * a.features + (lo - row0);

    // ---- loads that depend on nothing else (units without work read the first chunk's)
    const uint32_t off_c = a.offsets[c], off_c1 = a.offsets[c + 1];
    uint32_t x = behind ? a.mid_states[c * kStates + j] : a.states[c * kStates + j];
    const uint32_t len = a.lens[c * kStates + j];
    const uint32_t mid_len = split ? a.mid_lens[c * kStates + j] : 0u;
    const uint32_t lone = a.tb->lone;

    // ---- the words of the wave's chunks
    const uint64_t aligned0 = (static_cast<uint64_t>(off_c) * 2) & ~static_cast<uint64_t>(15);
    const uint32_t piece = live ? static_cast<uint32_t>((static_cast<uint64_t>(off_c1) * 2 - aligned0 + 15) & ~static_cast<uint64_t>(15)) : 0u;
    uint32_t place = 0, all = 0;
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r) {
        const uint32_t p = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(piece), static_cast<int>(r * kStates)));
        place += r < lane / kStates ? p : 0u;
        all += p;
    }
    const bool staged = all + 16 <= kEmbWindow;
    uint8_t *window = lds.stage + wave * kEmbWindow;
    if (staged) {
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
            auto of_unit = [&](uint32_t v) {
                return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), static_cast<int>(r * kStates)));
            };
            const uint64_t at = of_unit(static_cast<uint32_t>(aligned0)) |
                                (static_cast<uint64_t>(of_unit(static_cast<uint32_t>(aligned0 >> 32))) << 32);
            const uint32_t bytes = of_unit(piece);
            const uint4 *from = reinterpret_cast<const uint4 *>(reinterpret_cast<const uint8_t *>(a.words) + at);
            uint8_t *to = window + of_unit(place);
            for (uint32_t i = 0; i * 16 < bytes; i += 64)
                if ((i + lane) * 16 < bytes)
                    copy_to_lds(from + i + lane, to + i * 16);
        }
    }
    // ---- the slot table, beside it: the blob's, or made from its steps
    if (holds_table(a.n_chunks)) {
        for (uint32_t i = tid; i < kM / 4; i += THREADS)
            reinterpret_cast<uint4 *>(lds.lut)[i] = reinterpret_cast<const uint4 *>(a.tb->lut)[i];
    } else {
        const uint32_t begins[2] = {a.tb->step_of[tid], THREADS < kM / 8 ? a.tb->step_of[tid + THREADS < kM / 8 ? tid + THREADS : 0u] : 0u};
        for (uint32_t i = tid; i < kSteps / 4; i += THREADS)
            reinterpret_cast<uint4 *>(lds.steps)[i] = reinterpret_cast<const uint4 *>(a.tb->steps)[i];
        lds_barrier();
        if (lone >= 256)
            make_table(lds.steps, begins, a.tb, lds.lut);
    }
    wait_for_memory_acks();  // the words
    __syncthreads();

    // a row of its own for a token that is none
    if (unit < a.units && !valid && part == 0)
        for (uint32_t i = j; i < a.features / kRun; i += kStates)
            reinterpret_cast<uint4 *>(a.out + static_cast<uint64_t>(t) * a.features)[i] = make_uint4(0, 0, 0, 0);

    const uint32_t before = row_scan_u32(len) - len + (behind ? mid_len : 0u);
    const uint64_t run_byte = (static_cast<uint64_t>(off_c) + before) * 2;
    uint32_t most_turns = 0;
#pragma unroll
    for (uint32_t r = 0; r < 4; ++r)
        most_turns = max(most_turns, static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(turns), static_cast<int>(r * kStates))));
    const uint32_t from = begin + j * kRun;
    uint32_t wp = 0, wp_begin = 0;
    if (lone < 256) {
        embedding_walk<KB, true, NORM, EAGER>(lds.lut, NoWords{}, lone, x, wp, a, from, lo, hi, turns, most_turns, out);
    } else if (staged) {
        wp = wp_begin = wave * kEmbWindow + place + static_cast<uint32_t>(run_byte - aligned0);
        embedding_walk<KB, false, NORM, EAGER>(lds.lut, LdsWords{lds.stage}, 0u, x, wp, a, from, lo, hi, turns, most_turns, out);
    } else {
        const GlobalWords direct{reinterpret_cast<const uint8_t *>(a.words) + run_byte};
        embedding_walk<KB, false, NORM, false>(lds.lut, direct, 0u, x, wp, a, from, lo, hi, turns, most_turns, out);
    }
    // a walk that has come to the chunk's end or the entry points is checked there
    if (live && turns == (split ? kMidTurn : kTurns) && hi - begin == (1u << granule_shift)) {
        const uint32_t x_end = split && !behind ? a.mid_states[c * kStates + j] : kRansL;
        const uint32_t words_here = !split ? len : (behind ? len - mid_len : mid_len);
        if (x != x_end || wp - wp_begin != 2 * words_here)
            atomicOr(a.status, 1u);
    }
}

// ------------------------------------------------------------------------------------------
// Gradient:  grad[r] = bf16(scale * sum of g[t] over the tokens t with token[t] = r, in their order), every row of the table.
//
// Three launches, and nothing that depends on the order in which atomics arrive.
//   sort      the tokens in runs of 4096, each by one workgroup in LDS, by token and then position.  A run also tells where the
//             rows of each of 2048 ranges begin in it, and lists the pieces of 64 tokens that its longer segments consist of.
//   pieces    (more than 64 tokens) the sums of those pieces in binary32, so that a token that is very frequent is no workgroup's
//             work alone
//   write     a workgroup writes 16 KB of the gradient.  Two numbers per run tell whether any token belongs there; where none
//             does, which is nearly everywhere in a large table, it writes zeros.
// ------------------------------------------------------------------------------------------
constexpr uint32_t kSortRun = 4096, kSortThreads = 1024, kSortRanges = 2048;
constexpr uint32_t kPieceTokens = 64, kPiecesMost = 128;
struct SortedRun {
    uint32_t token[kSortRun];
    uint32_t index[kSortRun];            // position of the token in the call's tokens
    uint16_t piece_of[kSortRun];         // of the first token of a piece: its number
    uint16_t first[kSortRanges + 8];     // the first of a range of rows; first[kSortRanges]: how many there are
    uint16_t piece_at[kPiecesMost];
    uint16_t piece_tokens[kPiecesMost];
    uint32_t pieces;
    uint32_t pad[3];
};
static_assert(sizeof(SortedRun) % 16 == 0, "runs lie side by side");
// segments of more than 64 of 4096 tokens: at most 63, with at most 64 whole pieces and one more each
static_assert(kSortRun / kPieceTokens + (kSortRun - 1) / (kPieceTokens + 1) <= kPiecesMost, "room for all pieces");

struct EmbeddingGradArgs {
    const int64_t *tokens;
    uint64_t count;
    const uint16_t *grad_out;
    uint16_t *grad;
    SortedRun *runs;
    float *partial;        // [run][piece][features]
    uint32_t n_runs, rows, features;
    uint32_t range_shift;  // rows of a range: 1 << range_shift
    Divisor row_pieces;    // features / 8
    float scale;
};

__global__ __launch_bounds__(kSortThreads) void embedding_sort_kernel(const EmbeddingGradArgs a)
{
    __shared__ uint64_t keys[kSortRun];  // row << 12 | position in the run; a token that is none counts as row `rows`
    __shared__ uint32_t wave_sums[kSortThreads / 64];
    const uint32_t tid = threadIdx.x;
    const uint64_t base = static_cast<uint64_t>(blockIdx.x) * kSortRun;
    const uint32_t here = a.count - base < kSortRun ? static_cast<uint32_t>(a.count - base) : kSortRun;
    SortedRun &run = a.runs[blockIdx.x];
    uint32_t padded = 1;
    while (padded < here)
        padded *= 2;
    for (uint32_t i = tid; i < padded; i += kSortThreads) {
        uint64_t key = ~0ull;
        if (i < here) {
            const int64_t token = a.tokens[base + i];
            const uint64_t row = token >= 0 && token < static_cast<int64_t>(a.rows) ? static_cast<uint64_t>(token) : a.rows;
            key = row << 12 | i;
        }
        keys[i] = key;
    }
    __syncthreads();
    // bitonic sort (keys are distinct, so its result is the stable one)
    for (uint32_t size = 2; size <= padded; size *= 2) {
        for (uint32_t apart = size / 2; apart > 0; apart /= 2) {
            for (uint32_t i = tid; i < padded / 2; i += kSortThreads) {
                const uint32_t at = 2 * i - (i & (apart - 1)), other = at + apart;
                const uint64_t p = keys[at], q = keys[other];
                if ((p > q) == ((at & size) == 0)) {
                    keys[at] = q;
                    keys[other] = p;
                }
            }
            __syncthreads();
        }
    }
    // the first key that is not below `key`
    auto lower = [&](uint64_t key) {
        uint32_t low = 0, high = here;
        while (low < high) {
            const uint32_t mid = (low + high) / 2;
            if (keys[mid] < key)
                low = mid + 1;
            else
                high = mid;
        }
        return low;
    };
    const uint32_t valid = lower(static_cast<uint64_t>(a.rows) << 12);
    for (uint32_t i = tid; i < valid; i += kSortThreads) {
        run.token[i] = static_cast<uint32_t>(keys[i] >> 12);
        run.index[i] = static_cast<uint32_t>(base) + (static_cast<uint32_t>(keys[i]) & (kSortRun - 1));
    }
    for (uint32_t i = tid; i <= kSortRanges; i += kSortThreads) {
        const uint64_t row = static_cast<uint64_t>(i) << a.range_shift;
        run.first[i] = static_cast<uint16_t>(row >= a.rows ? valid : lower(row << 12));
    }
    // ---- pieces of the longer segments: four neighbouring places to a thread
    uint32_t starts = 0, lens[4] = {0, 0, 0, 0};
    if (valid > kPieceTokens) {
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k) {
            const uint32_t i = tid * 4 + k;
            if (i >= valid)
                break;
            const uint64_t row = keys[i] >> 12;
            const uint32_t low = lower(row << 12);
            if ((i - low) % kPieceTokens == 0 && low + kPieceTokens < valid && keys[low + kPieceTokens] >> 12 == row) {
                const uint32_t end = lower((row + 1) << 12);
                lens[k] = end - i < kPieceTokens ? end - i : kPieceTokens;
                ++starts;
            }
        }
    }
    const uint32_t upto = wave_scan_u32(starts, 0u, OpAdd{});
    if (tid % 64 == 63)
        wave_sums[tid / 64] = upto;
    __syncthreads();
    uint32_t number = upto - starts, total = 0;
    for (uint32_t w = 0; w < kSortThreads / 64; ++w) {
        number += w < tid / 64 ? wave_sums[w] : 0u;
        total += wave_sums[w];
    }
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k)
        if (lens[k]) {
            const uint32_t i = tid * 4 + k;
            run.piece_of[i] = static_cast<uint16_t>(number);
            run.piece_at[number] = static_cast<uint16_t>(i);
            run.piece_tokens[number] = static_cast<uint16_t>(lens[k]);
            ++number;
        }
    if (tid == 0)
        run.pieces = total;
}

// eight neighbouring elements added to their sums
__device__ __forceinline__ void add_eight(float (&sum)[8], const uint4 &v)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        sum[2 * p] += __uint_as_float(d[p] << 16);
        sum[2 * p + 1] += __uint_as_float(d[p] & 0xFFFF0000u);
    }
}

// The rows of grad_out that sorted places at .. at + count - 1 name, in that order; eight requested at a time.
__device__ __forceinline__ void add_rows(float (&sum)[8], const uint32_t *__restrict__ index, uint32_t count,
                                         const uint4 *__restrict__ grad_out, uint32_t row_pieces, uint32_t piece)
{
    constexpr uint32_t kTogether = 8;
    for (uint32_t s = 0; s < count; s += kTogether) {
        uint4 v[kTogether];
#pragma unroll
        for (uint32_t r = 0; r < kTogether; ++r)
            v[r] = grad_out[static_cast<uint64_t>(index[s + r < count ? s + r : s]) * row_pieces + piece];
#pragma unroll
        for (uint32_t r = 0; r < kTogether; ++r)
            if (s + r < count)
                add_eight(sum, v[r]);
    }
}

constexpr uint32_t kGradThreads = 256;
__global__ __launch_bounds__(kGradThreads) void embedding_pieces_kernel(const EmbeddingGradArgs a)
{
    const SortedRun &run = a.runs[blockIdx.y];
    const uint32_t number = blockIdx.x;
    if (number >= run.pieces)
        return;
    const uint32_t piece = blockIdx.z * kGradThreads + threadIdx.x;
    if (piece >= a.row_pieces.by)
        return;
    float sum[8] = {};
    add_rows(sum, run.index + run.piece_at[number], run.piece_tokens[number], reinterpret_cast<const uint4 *>(a.grad_out), a.row_pieces.by, piece);
    float4 *to = reinterpret_cast<float4 *>(a.partial + (static_cast<uint64_t>(blockIdx.y) * kPiecesMost + number) * a.features) + 2 * piece;
    to[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    to[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
}

constexpr uint32_t kGradPieces = 4;  // of 16 bytes, a thread's
__global__ __launch_bounds__(kGradThreads) void embedding_write_kernel(const EmbeddingGradArgs a)
{
    // (pieces of the table: fewer than 2^29)
    const uint32_t all = a.rows * a.row_pieces.by, from = blockIdx.x * (kGradThreads * kGradPieces);
    const uint32_t last = min(from + kGradThreads * kGradPieces, all) - 1;
    const uint32_t range0 = a.row_pieces.quotient(from) >> a.range_shift, range1 = (a.row_pieces.quotient(last) >> a.range_shift) + 1;
    uint4 *grad = reinterpret_cast<uint4 *>(a.grad);
    bool any = false;
    for (uint32_t r = 0; r < a.n_runs && !any; ++r)
        any = a.runs[r].first[range0] < a.runs[r].first[range1];
    if (!any) {
#pragma unroll
        for (uint32_t k = 0; k < kGradPieces; ++k)
            if (from + k * kGradThreads + threadIdx.x < all)
                grad[from + k * kGradThreads + threadIdx.x] = make_uint4(0, 0, 0, 0);
        return;
    }
    for (uint32_t k = 0; k < kGradPieces; ++k) {
        const uint32_t at = from + k * kGradThreads + threadIdx.x;
        if (at >= all)
            return;
        const uint32_t row = a.row_pieces.quotient(at), piece = at - row * a.row_pieces.by;
        float sum[8] = {};
        for (uint32_t r = 0; r < a.n_runs; ++r) {
            const SortedRun &run = a.runs[r];
            uint32_t low = run.first[row >> a.range_shift], high = run.first[(row >> a.range_shift) + 1];
            const uint32_t end = high;
            while (low < high) {
                const uint32_t mid = (low + high) / 2;
                if (run.token[mid] < row)
                    low = mid + 1;
                else
                    high = mid;
            }
            uint32_t upto = low;
            if (low + kPieceTokens < end && run.token[low + kPieceTokens] == row) {
                // a longer segment: its pieces, in order
                for (uint32_t number = run.piece_of[low];; ++number) {
                    const float4 *v = reinterpret_cast<const float4 *>(a.partial + (static_cast<uint64_t>(r) * kPiecesMost + number) * a.features) + 2 * piece;
                    const float4 p = v[0], q = v[1];
                    sum[0] += p.x;
                    sum[1] += p.y;
                    sum[2] += p.z;
                    sum[3] += p.w;
                    sum[4] += q.x;
                    sum[5] += q.y;
                    sum[6] += q.z;
                    sum[7] += q.w;
                    if (run.piece_tokens[number] < kPieceTokens || upto + kPieceTokens >= end || run.token[upto + kPieceTokens] != row)
                        break;
                    upto += kPieceTokens;
                }
            } else {
                while (upto < end && run.token[upto] == row)
                    ++upto;
                add_rows(sum, run.index + low, upto - low, reinterpret_cast<const uint4 *>(a.grad_out), a.row_pieces.by, piece);
            }
        }
        uint32_t d[4];
#pragma unroll
        for (int p = 0; p < 4; ++p)
            d[p] = bf16_of(sum[2 * p] * a.scale) | (bf16_of(sum[2 * p + 1] * a.scale) << 16);
        grad[at] = make_uint4(d[0], d[1], d[2], d[3]);
    }
}

}  // namespace nz
