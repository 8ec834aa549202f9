// Embedding on a compressed table for gfx950: rows decoded by token, and the table's gradient.
#pragma once

#include <type_traits>

#include "neuzip_format.h"
#include "neuzip_walk.h"

namespace nz {

// ------------------------------------------------------------------------------------------
// Lookup:  out[t] = bf16(scale * W_hat[token[t]]).
//
// A row lies in one chunk or in neighbouring ones, somewhere in it, and a state is decoded from its beginning or its entry point
// on.  So the unit of work is a row's share of one chunk (of half a chunk, where the blob has entry points): 16 lanes walk the
// chunk's 16 states up to the last turn that the row needs and leave the turns that belong to it, 16 bytes per lane and turn.  A wave
// takes four units.  Each copies its chunk's words straight into its wave's window of LDS, beside the slot table that the workgroup's
// waves share.
// Bound by the chain of a state's steps, 256 of 116 cycles each (12.4 us) where the blob has no entry points, whatever the number of
// tokens: 128256 x 4096, one token 16.7 us, 4096 tokens, 47 MB moved, 20.6; 777 of 50021 x 1160, k = 3, 20.1.  So a workgroup is small as
// long as that gives every CU one, and what does not depend on the tokens is requested before they are read.
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

// WHOLE: every unit of the wave is a whole chunk (or half of one), and all of it belongs to the row; turns is the same for all.
template <int KB, bool LONE, bool NORM, bool EAGER, bool WHOLE, class WordSrc>
__device__ __forceinline__ void embedding_walk(const uint32_t *__restrict__ lut, const WordSrc &src, uint32_t lone, uint32_t &x,
                                               uint32_t &wp, const EmbeddingArgs &a, uint32_t from, uint32_t lo, uint32_t hi,
                                               uint32_t turns, uint32_t most_turns, uint16_t *__restrict__ out)
{
    // this lane's runs begin at from, from + 128, ...; those inside lo .. hi - 1 belong to the row, whose part here goes to out
    uint32_t next = LONE ? 0u : src.peek(wp);
    auto request = [&](uint32_t q) {
        const uint32_t at = from + q * kTurn;
        const uint32_t here = WHOLE ? at : max(lo, min(at, hi - kRun));  // (some run of the row)
        uint64_t f = load_fields<KB>(a.sm, here);
        if constexpr (NORM)
            f |= static_cast<uint64_t>(a.coef[here >> a.block_shift]) << 32;
        return f;
    };
    uint64_t fields[kEmbAhead] = {};
    if (WHOLE || turns > 0)
#pragma unroll
        for (uint32_t r = 0; r < kEmbAhead; ++r)
            fields[r] = request(r);
    for (uint32_t q0 = 0; q0 < most_turns; q0 += kEmbAhead) {
        uint64_t ahead[kEmbAhead] = {};
        if (WHOLE || q0 + kEmbAhead < turns)
#pragma unroll
            for (uint32_t r = 0; r < kEmbAhead; ++r)
                ahead[r] = request(WHOLE && q0 + kEmbAhead >= most_turns ? r : q0 + kEmbAhead + r);  // (behind the last: the first again)
#pragma unroll
        for (uint32_t r = 0; r < kEmbAhead; ++r) {
            const uint32_t at = from + (q0 + r) * kTurn;
            // (lanes whose own unit is done go on with the wave's, to no effect: a state that is fed what is not its own stays in
            // the table, and reads at most a word per symbol)
            if (WHOLE || q0 + r < most_turns) {
                uint32_t e[8];
#pragma unroll
                for (int t = 0; t < 8; ++t)
                    e[t] = LONE ? lone : rans_get<EAGER>(lut, x, wp, next, src);
                if (WHOLE || at - lo < hi - lo) {
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
        uint8_t stage[kWaves * kEmbWindow];  // first: on 16 bytes, as direct copies need it
        uint32_t lut[kM];
        uint32_t steps[kSteps];
    } lds;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, j = tid & (kStates - 1);
    const uint32_t wave = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(tid >> 6)));
    const bool split = a.mid_states != nullptr;
    const uint32_t granule_shift = split ? 11u : 12u;
    static_assert(kChunk == 1u << 12 && kMidTurn * kTurn == 1u << 11, "log2 of a unit's elements");

    fetch_arguments(a);
    // ---- the tensor's table: the blob's slot table, or the steps that it is made from.  Nothing else depends on it, and it on nothing.
    const bool make_lut = !holds_table(a.n_chunks);
    constexpr uint32_t kTablePieces = kM / 4 / THREADS;  // of 16 bytes, a thread's
    uint4 table_piece[kTablePieces];
    const uint32_t begins[2] = {make_lut ? a.tb->step_of[tid] : 0u, make_lut && THREADS < kM / 8 ? a.tb->step_of[(tid + THREADS) % (kM / 8)] : 0u};
#pragma unroll
    for (uint32_t r = 0; r < kTablePieces; ++r) {
        const uint32_t i = tid + r * THREADS;
        table_piece[r] = make_uint4(0, 0, 0, 0);
        if (!make_lut)
            table_piece[r] = reinterpret_cast<const uint4 *>(a.tb->lut)[i];
        else if (i < kSteps / 4)
            table_piece[r] = reinterpret_cast<const uint4 *>(a.tb->steps)[i];
    }

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
    // (of a unit without work: 0, and no run lies in lo .. hi - 1)
    const uint32_t hi = live ? static_cast<uint32_t>(min(static_cast<uint64_t>(row1), first + (1ull << granule_shift))) : 0u;
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
    // ---- the slot table, beside it
    if (make_lut) {
#pragma unroll
        for (uint32_t r = 0; r < kTablePieces; ++r)
            if (tid + r * THREADS < kSteps / 4)
                reinterpret_cast<uint4 *>(lds.steps)[tid + r * THREADS] = table_piece[r];
        lds_barrier();
        if (lone >= 256)
            make_table(lds.steps, begins, a.tb, lds.lut);
    } else {
#pragma unroll
        for (uint32_t r = 0; r < kTablePieces; ++r)
            reinterpret_cast<uint4 *>(lds.lut)[tid + r * THREADS] = table_piece[r];
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
    const bool whole = __all(!live || (lo == begin && hi - begin == (1u << granule_shift)));
    if (lone < 256) {
        embedding_walk<KB, true, NORM, EAGER, false>(lds.lut, NoWords{}, lone, x, wp, a, from, lo, hi, turns, most_turns, out);
    } else if (staged) {
        wp = wp_begin = wave * kEmbWindow + place + static_cast<uint32_t>(run_byte - aligned0);
        if (!whole)
            embedding_walk<KB, false, NORM, EAGER, false>(lds.lut, LdsWords{lds.stage}, 0u, x, wp, a, from, lo, hi, turns, most_turns, out);
        else if (live)
            embedding_walk<KB, false, NORM, EAGER, true>(lds.lut, LdsWords{lds.stage}, 0u, x, wp, a, from, lo, hi, turns, most_turns, out);
    } else {
        const GlobalWords direct{reinterpret_cast<const uint8_t *>(a.words) + run_byte};
        embedding_walk<KB, false, NORM, false, false>(lds.lut, direct, 0u, x, wp, a, from, lo, hi, turns, most_turns, out);
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
// Three launches (few tokens: one, see embedding_few_kernel), and nothing that depends on the order in which atomics arrive.
//   sort      the tokens in runs of 4096, by token and then position: an element's place is the number of those that come before it,
//             which is counted, 32 elements to a workgroup, so that a run is sorted by many CUs in one go (one workgroup with a
//             bitonic network in LDS took 45 us for 4096 tokens).  Counted the same way: where the rows of each of 2048 ranges begin
//             in the run.
//   pieces    a row whose tokens pass the end of a block of 64 sorted places is summed block by block, in
//             binary32, so that a token that is very frequent is no workgroup's work alone
//   rows      a workgroup to a row with tokens, at the first of them, adds its tokens up, or its pieces, and stores it.
// Most of the work for a large table is zeros: the first launch's other workgroups fill the gradient with them meanwhile (4096
// tokens, 128256 x 4096: 159 us, in which the sort is done after 11; three quarters of the zeros beside the second launch gave nothing).
// Bound by memory there, 1.05 GB at 6.5 TB/s, the pieces' 12 and the rows' 20 us behind it: 186 to 193 us; by latency and launches with
// small tables (5003 x 520: 7.2, 6.5 and 5.0 us), which is why few tokens go another way.
// ------------------------------------------------------------------------------------------
constexpr uint32_t kSortRun = 4096, kSortRanges = 2048, kSortQueries = 32;
constexpr uint32_t kBlockTokens = 64, kBlocks = kSortRun / kBlockTokens;
constexpr uint32_t kPieces = 2 * kBlocks;  // of a run: of a row that began before the block; of one that begins in it and passes its end
struct SortedRun {
    uint32_t token[kSortRun];
    uint32_t index[kSortRun];         // position of the token in the call's tokens
    uint32_t first[kSortRanges + 4];  // the first of a range of rows; first[kSortRanges]: how many there are
};
static_assert(sizeof(SortedRun) % 16 == 0, "runs lie side by side");

struct EmbeddingGradArgs {
    const int64_t *tokens;
    uint64_t count;
    const uint16_t *grad_out;
    uint16_t *grad;
    SortedRun *runs;
    float *partial;        // [run][piece][features]
    uint32_t n_runs, rows, features;
    uint32_t sort_wgs;     // workgroups that sort a run
    uint32_t range_shift;  // rows of a range: 1 << range_shift
    Divisor row_pieces;    // features / 8
    float scale;
};

template <uint32_t THREADS>
__global__ __launch_bounds__(THREADS) void embedding_sort_kernel(const EmbeddingGradArgs a)
{
    const uint32_t sorting = a.sort_wgs * a.n_runs;
    if (blockIdx.x >= sorting) {
        // Zeros, 16 bytes to a thread: 1.05 GB take 155 us, with four or sixteen times as much 177 and 191.  (Fewer than 2^29 pieces.)
        const uint32_t piece = (blockIdx.x - sorting) * THREADS + threadIdx.x;
        if (piece < a.rows * a.row_pieces.by)
            reinterpret_cast<uint4 *>(a.grad)[piece] = make_uint4(0, 0, 0, 0);
        return;
    }
    const uint32_t of_run = a.sort_wgs == 0 ? 0u : blockIdx.x / a.sort_wgs, group = blockIdx.x - of_run * a.sort_wgs;
    // Queries are the run's elements, then the ranges' first rows.  A wave's lanes hold the 32 queries twice, for the two parts of the run
    // that are the wave's (of 8 parts in a workgroup of 256 threads, of 32 in one of 1024).
    constexpr uint32_t kParts = THREADS / kSortQueries;
    __shared__ __align__(16) uint32_t rows[kSortRun];
    __shared__ uint32_t before[kSortQueries];
    const uint32_t tid = threadIdx.x, query = tid % kSortQueries, part = tid / kSortQueries;
    const uint64_t base = static_cast<uint64_t>(of_run) * kSortRun;
    const uint32_t here = a.count - base < kSortRun ? static_cast<uint32_t>(a.count - base) : kSortRun;
    const uint32_t padded = (here + 4 * kParts - 1) / (4 * kParts) * (4 * kParts), each = padded / kParts;
    // (all of a thread's tokens requested together)
    constexpr uint32_t kEach = kSortRun / THREADS;
    int64_t tokens[kEach];
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
        const uint32_t i = r * THREADS + tid;
        tokens[r] = i < here ? a.tokens[base + i] : -1;
    }
#pragma unroll
    for (uint32_t r = 0; r < kEach; ++r) {
        const uint32_t i = r * THREADS + tid;
        if (i < padded)  // (of no row: behind them all)
            rows[i] = tokens[r] >= 0 && tokens[r] < static_cast<int64_t>(a.rows) ? static_cast<uint32_t>(tokens[r]) : ~0u;
    }
    if (tid < kSortQueries)
        before[tid] = 0;
    __syncthreads();
    const uint32_t number = group * kSortQueries + query;
    const bool is_element = number < here;
    const uint32_t range = number - here;  // (of a query behind the elements)
    const uint64_t range_row = static_cast<uint64_t>(range) << a.range_shift;
    const uint32_t row = is_element ? rows[number] : (range_row < a.rows ? static_cast<uint32_t>(range_row) : a.rows);
    // Elements in front of this one come before it if their rows are not above its own, those behind if they are below it.
    const uint32_t not_above = is_element ? (row == ~0u ? row : row + 1) : row;
    const uint32_t p0 = group * kSortQueries;
    uint32_t count = 0;
#pragma unroll 8
    for (uint32_t j = part * each; j < (part + 1) * each; j += 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(rows + j);
        const uint32_t limit = j < p0 ? not_above : row;
        count += v.x < limit;
        count += v.y < limit;
        count += v.z < limit;
        count += v.w < limit;
    }
    // ... of the workgroup's own, those in front (the equal ones have not been counted)
    if (part == 0 && is_element) {
#pragma unroll
        for (uint32_t j = 0; j < kSortQueries; j += 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(rows + p0 + j);
            count += v.x == row && j < query;
            count += v.y == row && j + 1 < query;
            count += v.z == row && j + 2 < query;
            count += v.w == row && j + 3 < query;
        }
    }
    atomicAdd(&before[query], count);
    __syncthreads();
    if (tid >= kSortQueries)
        return;
    SortedRun &run = a.runs[of_run];
    const uint32_t place = before[tid];
    if (is_element) {
        if (row != ~0u) {
            run.token[place] = row;
            run.index[place] = static_cast<uint32_t>(base) + number;
        }
    } else if (range <= kSortRanges) {
        run.first[range] = place;
    }
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

// The rows of grad_out that sorted places at .. at + count - 1 name, in that order, sixteen requested at a time (count is the same for
// the workgroup).
constexpr uint32_t kGradThreads = 256;
__device__ __forceinline__ void add_rows(float (&sum)[8], const uint32_t *__restrict__ index, uint32_t count,
                                         const uint4 *__restrict__ grad_out, uint32_t row_pieces, uint32_t piece)
{
    auto take = [&](auto rows, uint32_t s) {
        constexpr uint32_t N = decltype(rows)::value;
        uint4 v[N];
#pragma unroll
        for (uint32_t r = 0; r < N; ++r)
            v[r] = grad_out[static_cast<uint64_t>(index[s + r]) * row_pieces + piece];
#pragma unroll
        for (uint32_t r = 0; r < N; ++r)
            add_eight(sum, v[r]);
    };
    uint32_t s = 0;
    for (; s + 16 <= count; s += 16)
        take(std::integral_constant<uint32_t, 16>{}, s);
    for (; s + 4 <= count; s += 4)
        take(std::integral_constant<uint32_t, 4>{}, s);
    for (; s < count; ++s)
        take(std::integral_constant<uint32_t, 1>{}, s);
}

__global__ __launch_bounds__(kGradThreads) void embedding_pieces_kernel(const EmbeddingGradArgs a)
{
    const SortedRun &run = a.runs[blockIdx.y];
    const uint32_t begin = blockIdx.x / 2 * kBlockTokens, valid = run.first[kSortRanges], lane = threadIdx.x % 64;
    const bool begins_here = blockIdx.x % 2;
    if (begin >= valid)
        return;
    const uint32_t end = min(begin + kBlockTokens, valid);
    const uint32_t before = begin > 0 ? run.token[begin - 1] : ~0u, behind = end < valid ? run.token[end] : ~0u;
    const uint32_t token = begin + lane < end ? run.token[begin + lane] : ~0u;
    // the row that began before the block, or the one that passes its end and is another
    const uint32_t row = begins_here ? behind : before;
    const uint64_t mine = __ballot(token == row && row != ~0u && (!begins_here || row != before));
    if (!mine)
        return;
    const uint32_t from = begin + static_cast<uint32_t>(__builtin_ctzll(mine)), count = static_cast<uint32_t>(__builtin_popcountll(mine));
    const uint32_t piece = blockIdx.z * kGradThreads + threadIdx.x;
    if (piece >= a.row_pieces.by)
        return;
    float sum[8] = {};
    add_rows(sum, run.index + from, count, reinterpret_cast<const uint4 *>(a.grad_out), a.row_pieces.by, piece);
    float4 *to = reinterpret_cast<float4 *>(a.partial + (static_cast<uint64_t>(blockIdx.y) * kPieces + blockIdx.x) * a.features) + 2 * piece;
    to[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    to[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
}

// run.token[...] of a row: the places from .. upto - 1
__device__ __forceinline__ void places_of(const SortedRun &run, uint32_t row, uint32_t range_shift, uint32_t &from, uint32_t &upto)
{
    uint32_t low = run.first[row >> range_shift], high = run.first[(row >> range_shift) + 1];
    const uint32_t end = high;
    while (low < high) {
        const uint32_t mid = (low + high) / 2;
        if (run.token[mid] < row)
            low = mid + 1;
        else
            high = mid;
    }
    from = low;
    high = end;
    while (low < high) {
        const uint32_t mid = (low + high) / 2;
        if (run.token[mid] <= row)
            low = mid + 1;
        else
            high = mid;
    }
    upto = low;
}

__device__ __forceinline__ void leave_row(const EmbeddingGradArgs &a, uint32_t row, uint32_t piece, const float (&sum)[8], float scale)
{
    uint32_t d[4];
#pragma unroll
    for (int p = 0; p < 4; ++p)
        d[p] = bf16_of(sum[2 * p] * scale) | (bf16_of(sum[2 * p + 1] * scale) << 16);
    reinterpret_cast<uint4 *>(a.grad)[static_cast<uint64_t>(row) * a.row_pieces.by + piece] = make_uint4(d[0], d[1], d[2], d[3]);
}

__global__ __launch_bounds__(kGradThreads) void embedding_rows_kernel(const EmbeddingGradArgs a)
{
    const uint32_t own = blockIdx.y, place = blockIdx.x, lane = threadIdx.x % 64;
    const SortedRun &run = a.runs[own];
    const uint32_t valid = run.first[kSortRanges];
    if (place >= valid)
        return;
    const uint32_t row = run.token[place];
    if (place > 0 && run.token[place - 1] == row)
        return;
    // the row's places in its own run: as many as follow the first without a gap, ...
    const uint32_t block = place / kBlockTokens, block_end = (block + 1) * kBlockTokens;
    const uint32_t next = place + 1 + lane < valid ? run.token[place + 1 + lane] : ~0u;
    const uint32_t corner = block_end + lane * kBlockTokens < valid ? run.token[block_end + lane * kBlockTokens] : ~0u;
    const uint64_t others = ~__ballot(next == row), others_far = ~__ballot(corner == row);
    const uint32_t follow = others ? static_cast<uint32_t>(__builtin_ctzll(others)) : 64u;
    // ... or the blocks whose ends it passes
    const uint32_t passes = others_far ? static_cast<uint32_t>(__builtin_ctzll(others_far)) : 64u;
    // a row that a run before this one has is that one's
    for (uint32_t r0 = 0; r0 < own; r0 += 64) {
        uint32_t from = 0, upto = 0;
        if (r0 + lane < own)
            places_of(a.runs[r0 + lane], row, a.range_shift, from, upto);
        if (__ballot(from < upto))
            return;
    }
    const uint32_t piece = blockIdx.z * kGradThreads + threadIdx.x;
    const bool live = piece < a.row_pieces.by;
    const uint4 *grad_out = reinterpret_cast<const uint4 *>(a.grad_out);
    float sum[8] = {};
    // the sums of the pieces that the places from `from` on are in, in order
    auto add_pieces = [&](uint32_t r, uint32_t from, uint32_t ends) {
        auto take = [&](auto pieces, uint32_t k) {
            constexpr uint32_t N = decltype(pieces)::value;
            float4 p[N], q[N];
#pragma unroll
            for (uint32_t n = 0; n < N; ++n) {
                const uint32_t number = 2 * (from / kBlockTokens + k + n) + (k + n == 0 ? 1 : 0);
                const float4 *v = reinterpret_cast<const float4 *>(a.partial + (static_cast<uint64_t>(r) * kPieces + number) * a.features) + 2 * piece;
                p[n] = v[0];
                q[n] = v[1];
            }
#pragma unroll
            for (uint32_t n = 0; n < N; ++n) {
                sum[0] += p[n].x;
                sum[1] += p[n].y;
                sum[2] += p[n].z;
                sum[3] += p[n].w;
                sum[4] += q[n].x;
                sum[5] += q[n].y;
                sum[6] += q[n].z;
                sum[7] += q[n].w;
            }
        };
        uint32_t k = 0;
        for (; k + 8 <= ends + 1; k += 8)
            take(std::integral_constant<uint32_t, 8>{}, k);
        for (; k <= ends; ++k)
            take(std::integral_constant<uint32_t, 1>{}, k);
    };
    if (live) {
        if (passes)
            add_pieces(own, place, passes);
        else
            add_rows(sum, run.index + place, 1 + follow, grad_out, a.row_pieces.by, piece);
    }
    // ... and in the runs behind it, a run to a lane
    for (uint32_t r0 = own + 1; r0 < a.n_runs; r0 += 64) {
        uint32_t from = 0, upto = 0;
        if (r0 + lane < a.n_runs)
            places_of(a.runs[r0 + lane], row, a.range_shift, from, upto);
        for (uint64_t left = __ballot(from < upto); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const uint32_t begin = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(from), l));
            const uint32_t end = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(upto), l));
            const uint32_t ends = (end - 1) / kBlockTokens - begin / kBlockTokens;
            if (live) {
                if (ends)
                    add_pieces(r0 + l, begin, ends);
                else
                    add_rows(sum, a.runs[r0 + l].index + begin, end - begin, grad_out, a.row_pieces.by, piece);
            }
        }
    }
    if (live)
        leave_row(a, row, piece, sum, a.scale);
}

// Few tokens in one launch: a thread to 16 bytes of the gradient.  Every wave looks its tokens over, a lane to each; those of the workgroup's
// rows are added in their order, several requested at a time, by the threads whose row they name.
//   PARTS 1   up to 64 tokens, all of them every wave's
//   PARTS 4   up to 512: a workgroup holds a quarter as much of the gradient, its waves have a quarter of the tokens each, and the first adds
//             their sums up in order
// A row without tokens is left as zeros, whatever the factor: a negative one would make them -0, an infinity or a NaN a NaN.
template <int PARTS>
__global__ __launch_bounds__(kGradThreads) void embedding_few_kernel(const EmbeddingGradArgs a)
{
    constexpr uint32_t kWide = kGradThreads / PARTS, kChunks = PARTS == 1 ? 1 : 2, kAtOnce = PARTS == 1 ? 8 : 16;
    const uint32_t tid = threadIdx.x, lane = tid % 64, row_pieces = a.row_pieces.by;
    const uint32_t part = PARTS == 1 ? 0u : tid / 64, at = PARTS == 1 ? tid : lane;
    const uint32_t flat0 = blockIdx.x * kWide, flat = flat0 + at;  // (fewer than 2^29 pieces)
    const uint32_t first = a.row_pieces.quotient(flat0), own_rows = a.row_pieces.quotient(flat0 + kWide - 1) - first + 1;
    const uint32_t row = a.row_pieces.quotient(flat), own = row - first, piece = flat - row * row_pieces;
    const bool live = row < a.rows;
    const uint32_t count = static_cast<uint32_t>(a.count), each = (count + PARTS - 1) / PARTS, begin = part * each;
    uint64_t off[kChunks];
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) {
        const uint32_t in_part = c * 64 + lane;
        const int64_t token = in_part < each && begin + in_part < count ? a.tokens[begin + in_part] : -1;
        off[c] = token < static_cast<int64_t>(a.rows) ? static_cast<uint64_t>(token) - first : ~0ull;  // (a token below them is far behind)
    }
    float sum[8] = {};
    bool mine = false;  // a token names the thread's row
#pragma unroll
    for (uint32_t c = 0; c < kChunks; ++c) {
        uint64_t left = __ballot(off[c] < own_rows);
        while (left) {
            uint4 v[kAtOnce];
#pragma unroll
            for (uint32_t n = 0; n < kAtOnce; ++n) {
                const uint32_t l = left ? static_cast<uint32_t>(__builtin_ctzll(left)) : 0u;
                const uint32_t of = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(static_cast<uint32_t>(off[c])), static_cast<int>(l)));
                v[n] = make_uint4(0, 0, 0, 0);
                const bool here = live && left && of == own;
                mine = mine || here;
                if (here)
                    v[n] = reinterpret_cast<const uint4 *>(a.grad_out)[static_cast<uint64_t>(begin + c * 64 + l) * row_pieces + piece];
                left &= left - 1;  // (of none: none)
            }
#pragma unroll
            for (uint32_t n = 0; n < kAtOnce; ++n)
                add_eight(sum, v[n]);
        }
    }
    if constexpr (PARTS > 1) {
        __shared__ float4 sums[PARTS][2][64];
        __shared__ uint64_t has[PARTS];  // the lanes with a token in that part
        const uint64_t lanes = __ballot(mine);
        if (lanes) {
            sums[part][0][lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            sums[part][1][lane] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        }
        if (lane == 0)
            has[part] = lanes;
        __syncthreads();
        if (part > 0)
            return;
#pragma unroll
        for (uint32_t p = 1; p < PARTS; ++p) {
            if (!has[p])
                continue;
            mine = mine || (has[p] >> lane & 1u);
            const float4 u = sums[p][0][lane], v = sums[p][1][lane];
            sum[0] += u.x;
            sum[1] += u.y;
            sum[2] += u.z;
            sum[3] += u.w;
            sum[4] += v.x;
            sum[5] += v.y;
            sum[6] += v.z;
            sum[7] += v.w;
        }
    }
    if (live)
        leave_row(a, row, piece, sum, mine ? a.scale : 0.0f);
}

}  // namespace nz
