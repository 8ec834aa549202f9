// Gated feed-forward block on dense bf16 weights for gfx950:  h = act(x Wg^T) * (x Wu^T)  and its gradients, as products of
// matrices in the matrix cores.
//
// One kernel serves all of them.  It computes  C[i][j] = sum over k of Q(i, k) P(j, k)  for a tile of i and j at a time, the sums
// in binary32:
//   kForward     C = x Wg^T and x Wu^T side by side: half of a tile's j are rows of Wg, the other half the same rows of Wu, so
//                that a lane holds both sums of an output and leaves h (and, for the backward pass, both sums) by itself
//   kInputGrad   dx = dg Wg + du Wu, one sum over the 2 x out_features of both
//   kWeightGrad  dWg = dg^T x and dWu = du^T x, sums over the tokens; half of the tiles are the one's, half the other's
// The operand that supplies i or j lies with k along its rows (x and the weights in kForward, dg and du in kInputGrad), or with k
// down its columns (the others).
//
// Measured, 2048 tokens, 4096 -> 2 x 14336 (481 * 10^9 operations each): forward with both sums kept 398 to 416 us, input gradient 334 to 356
// and 13 for its slices, weight gradients 387 to 414; forward of 1000 tokens 184 = 1277 TFLOP/s.  The matrix cores are busy in 0.56 to 0.72 of the cycles; with
// operands of zeros, and the clock at 2.4 instead of 2.0 GHz, the same launches take 15 to 25 % less: power is what bounds them.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>
#include <type_traits>

#include "neuzip_gated_shape.h"

namespace nz {

struct GatedArgs {
    const uint16_t *q[2];   // kForward: x, x;  kInputGrad: dg, du;  kWeightGrad: dg, du
    const uint16_t *p[2];   // Wg, Wu;  Wg, Wu;  x, x
    uint16_t *c[2];         // h, -;  dx, -;  dWg, dWu
    float *gate, *up;       // kForward: the two sums, for the backward pass (nullptr: they are not kept)
    float *partial;         // kInputGrad, several slices: the sums of a slice leave as they are, to partial[slice][i][j]
    uint32_t rows;          // i: tokens, tokens, out_features
    uint32_t cols;          // j: out_features, in_features, in_features
    uint32_t depth;         // k: in_features, out_features (of each half), tokens
    uint32_t q_row, p_row, c_row;  // elements from one row to the next
    uint32_t tiles_i, tiles_j;     // of one half
    uint32_t slices;        // of k
    uint32_t activation;
};

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 gated_bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short gated_s16x4_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float gated_f32x4_t;

// ---- activations: act(g) = g * sigmoid(z(g)), z = g (SiLU) or 2 sqrt(2 / pi) (g + 0.044715 g^3) (GELU, tanh form)
constexpr float kGeluScale = 1.5957691216057308f;  // 2 sqrt(2 / pi)
__device__ __forceinline__ float gated_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ float gated_argument(float g, uint32_t activation)
{
    return activation ? kGeluScale * (g + 0.044715f * g * g * g) : g;
}
__device__ __forceinline__ float gated_value(float g, uint32_t activation)
{
    return g * gated_sigmoid(gated_argument(g, activation));
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
    typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
    const f32x2_t v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// 16 bytes per lane from memory straight into LDS, lane l's to M0 + OFFSET + 16 l.  Not the builtin: the compiler would wait for such
// a copy in front of the next read of LDS, whichever buffer it is from.  The waits are the caller's.  The offset counts on both
// sides, so the lane's address is given without it; up to four copies, 1 KB apart, share a place in M0 (between whose writing and the
// copy an instruction has to stand).
constexpr uint32_t kGatedShared = 4, kGatedBias = (kGatedShared - 1) * 1024;
__device__ __forceinline__ void gated_copy_place(uint32_t to) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(to)); }
template <uint32_t OFFSET>
__device__ __forceinline__ void gated_copy(const uint8_t *base, uint32_t offset)
{
    asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(offset), "s"(base), "n"(OFFSET));
}
template <uint32_t OFFSET>
__device__ __forceinline__ void gated_copy(const uint8_t *from)
{
    asm volatile("global_load_lds_dwordx4 %0, off offset:%1" ::"v"(from), "n"(OFFSET));
}

// All but the last PASS of the wave's copies have come, and everyone holds in registers what it has read of LDS so far.
template <uint32_t PASS>
__device__ __forceinline__ void gated_arrive(const uint8_t *lds)
{
    asm volatile("s_waitcnt vmcnt(%1) lgkmcnt(0)\n\ts_barrier" ::"v"(lds), "n"(PASS) : "memory");
}

// What lanes read that have no k of their own: zeros.
__device__ const uint4 kGatedZeros[1] = {};

// f(0), f(1), ... f(N - 1), each with its number known to the compiler
template <int N, int AT = 0, class F>
__device__ __forceinline__ void each_of(const F &f)
{
    if constexpr (AT < N) {
        f(std::integral_constant<uint32_t, AT>{});
        each_of<N, AT + 1>(f);
    }
}

// ---- one operand's tile in LDS: R values of i (or j) by 64 of k, R * 128 bytes.
// Along k: a row of the tile is 64 k, 128 bytes, 8 pieces of 16 bytes, piece p of row r in place p ^ (r / 2 % 8).
// Across k: a row is one k and its R values, in units of 16 values; unit u of row k in place u ^ f(k), f = k % 4 + 4 * (k / 8 % 2):
// the eight rows that half a wave reads a unit of at a time then lie in different banks.
template <int R, int WAVES, bool ALONG>
struct GatedOperand {
    static constexpr uint32_t kBytes = R * kGatedDepth * 2;
    static constexpr uint32_t kCopies = kBytes / 1024 / WAVES;  // a wave's, 1 KB each
    static constexpr uint32_t kPieces = R / 8;                  // ACROSS: of a row
    uint32_t offset[kCopies];  // of the lane's pieces in the tile's first step, less what the copy adds, plus kGatedBias
    uint32_t k_of;             // the k of the lane's piece in copy 0

    // left: values from the tile's first on (a lane that has none reads another's: nobody looks at the sums)
    __device__ __forceinline__ void set_up(uint32_t wave, uint32_t lane, uint32_t left, uint32_t row_elems)
    {
#pragma unroll
        for (uint32_t n = 0; n < kCopies; ++n) {
            const uint32_t copy = wave * kCopies + n, shift = kGatedBias - n % kGatedShared * 1024;
            if constexpr (ALONG) {
                uint32_t r = copy * 8 + lane / 8;
                const uint32_t piece = (lane % 8) ^ (r / 2 % 8);
                r = r < left ? r : left - 1;
                offset[n] = (r * row_elems + piece * 8) * 2 + shift;
                if (n == 0)
                    k_of = piece * 8;
            } else {
                const uint32_t k = copy * (64 / kPieces) + lane / kPieces;
                const uint32_t f = k % 4 + k / 8 % 2 * 4;
                uint32_t piece = (((lane % kPieces) / 2) ^ f) * 2 + lane % 2;
                piece = piece * 8 < left ? piece : 0u;
                offset[n] = (k * row_elems + piece * 8) * 2 + shift;
                if (n == 0)
                    k_of = k;
            }
        }
    }
    // requests copy N of the tile that begins at from + kGatedBias.  RAGGED: only `depth` of its k are there, the others are zeros.
    template <bool RAGGED, uint32_t N>
    __device__ __forceinline__ void request(const uint8_t *from, uint32_t to, uint32_t wave, uint32_t depth) const
    {
        if constexpr (N % kGatedShared == 0)
            gated_copy_place(to + (wave * kCopies + N) * 1024);
        constexpr uint32_t kOffset = N % kGatedShared * 1024;
        if constexpr (RAGGED) {
            // (along k, every other copy's rows hold their halves of 32 k the other way round)
            static_assert(kCopies % 2 == 0, "a wave's first copy is an even one");
            const uint32_t k = ALONG ? k_of ^ (N % 2 * 32) : k_of + N * (64 / kPieces);
            gated_copy<kOffset>(k < depth ? from + offset[N] : reinterpret_cast<const uint8_t *>(kGatedZeros) - kOffset);
        } else {
            gated_copy<kOffset>(from, offset[N]);
        }
    }
    // the lane's address of the operand's first 16 values (first: their number in the tile), for read()
    static __device__ __forceinline__ uint32_t lane_address(uint32_t first, uint32_t lane)
    {
        if constexpr (ALONG) {
            return (first + lane % 16) * 128 + (((lane / 16) ^ (lane % 16 / 2)) * 16);
        } else {
            const uint32_t i = lane % 16, g = lane / 16, f = i / 4 + (g % 2) * 4;
            return (8 * g + i / 4) * (R * 2) + ((first / 16) ^ f) * 32 + i % 4 * 8;
        }
    }
    // 16 values (the tile's `which`th from the first) by the 32 k of half `h`: lane l value l % 16, k = 8 * (l / 16) .. + 7
    static __device__ __forceinline__ gated_bf16x8_t read(const uint8_t *tile, uint32_t address, uint32_t which, uint32_t h)
    {
        if constexpr (ALONG) {
            return *reinterpret_cast<const gated_bf16x8_t *>(tile + (address ^ (h * 64)) + which * 2048);
        } else {
            typedef __attribute__((address_space(3))) gated_s16x4_t lds_s16x4_t;
            const uint8_t *at = tile + (address ^ (which * 32)) + h * 32 * (R * 2);
            union {
                gated_s16x4_t s[2];
                gated_bf16x8_t v;
            } u;
            u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(at));
            u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(at + 4 * (R * 2)));
            return u.v;
        }
    }
};

// Launch shape: tiles of SIZE i by SIZE j, four waves of SIZE / 2 by SIZE / 2.
constexpr uint32_t kGatedWaves = 4, kGatedThreads = kGatedWaves * 64;
// RING: the steps that LDS holds, of the operand for i; of the one for j one more.  Two and three are all of the 160 KB for a tile of 256,
// or half of them for one of 128, of which two share a CU.  Where there are fewer of those than CUs, nothing else hides the wait for memory,
// and four and five are held (two held, 4096 -> 4096, 200 tokens: forward 35.7 us, 29.7 so).
template <int SIZE, int RING>
__device__ __forceinline__ uint8_t *gated_lds()
{
    __shared__ __align__(16) uint8_t lds[(2 * RING + 1) * SIZE * kGatedDepth * 2];
    return lds;
}

// workgroup `index` of `all` that compute FORM
template <GatedForm FORM, int SIZE, int RING>
__device__ __forceinline__ void gated_workgroup(const GatedArgs &a, const uint32_t index, const uint32_t all)
{
    constexpr int WAVES = kGatedWaves;
    constexpr bool Q_ALONG = FORM != kWeightGrad, P_ALONG = FORM == kForward;
    constexpr int TILES = SIZE / 2 / 16;  // a wave has TILES x TILES sums of 16 x 16
    typedef GatedOperand<SIZE, WAVES, Q_ALONG> Q;
    typedef GatedOperand<SIZE, WAVES, P_ALONG> P;
    typedef GatedOperand<SIZE / 2, WAVES, true> Half;  // kForward: the rows of one weight
    constexpr uint32_t kQRing = RING, kPRing = RING + 1;
    constexpr uint32_t kQEnd = kQRing * Q::kBytes, kPEnd = kQEnd + kPRing * P::kBytes;
    uint8_t *const lds = gated_lds<SIZE, RING>();
    static_assert(kPEnd == (2 * RING + 1) * SIZE * kGatedDepth * 2, "as gated_lds() has it");

    const uint32_t lane = threadIdx.x % 64;
    const uint32_t wave = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x / 64)));
    // Which tile.  Workgroups go to the 8 XCDs in turn: each XCD takes a run of neighbouring tiles, and in it columns of 8 tiles of
    // i, so that what its L2 holds of both operands is used again.
    const uint32_t per = all / 8, more = all % 8, xcd = index % 8;
    uint32_t tile = xcd * per + (xcd < more ? xcd : more) + index / 8;
    const uint32_t per_slice = a.tiles_i * a.tiles_j * (FORM == kWeightGrad ? 2 : 1);
    const uint32_t slice = tile / per_slice;
    tile -= slice * per_slice;
    const uint32_t half = FORM == kWeightGrad ? tile / (a.tiles_i * a.tiles_j) : 0u;
    tile -= half * (a.tiles_i * a.tiles_j);
    constexpr uint32_t kBand = 8;
    const uint32_t band = tile / (kBand * a.tiles_j), in_band = tile - band * (kBand * a.tiles_j);
    const uint32_t band_rows = a.tiles_i - band * kBand < kBand ? a.tiles_i - band * kBand : kBand;
    const uint32_t ti = band * kBand + in_band % band_rows, tj = in_band / band_rows;
    // kForward: a tile's j are SIZE / 2 outputs, of both weights
    constexpr uint32_t kTileJ = FORM == kForward ? SIZE / 2 : SIZE;
    const uint32_t i0 = ti * SIZE, j0 = tj * kTileJ;

    // ---- what this wave copies
    Q q;
    P p;
    q.set_up(wave, lane, a.rows - i0, a.q_row);
    const uint8_t *q_base[2], *p_base[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        q_base[h] = reinterpret_cast<const uint8_t *>(a.q[h]) + static_cast<uint64_t>(i0) * (Q_ALONG ? a.q_row : 1u) * 2;
        p_base[h] = reinterpret_cast<const uint8_t *>(a.p[h]) + static_cast<uint64_t>(j0) * (P_ALONG ? a.p_row : 1u) * 2;
    }
    Half half_p;
    if constexpr (FORM == kForward)
        half_p.set_up(wave, lane, a.cols - j0, a.p_row);
    else
        p.set_up(wave, lane, a.cols - j0, a.p_row);

    // ---- steps of 64 k: all of one half, then (kInputGrad) all of the other
    const uint32_t half_steps = (a.depth + kGatedDepth - 1) / kGatedDepth;
    const uint32_t steps_all = FORM == kInputGrad ? 2 * half_steps : half_steps;
    const uint32_t s_begin = static_cast<uint32_t>(static_cast<uint64_t>(steps_all) * slice / a.slices);
    const uint32_t steps = static_cast<uint32_t>(static_cast<uint64_t>(steps_all) * (slice + 1) / a.slices) - s_begin;
    // what is requested next
    const uint32_t lds_at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t *)lds));
    const uint64_t q_step = static_cast<uint64_t>(kGatedDepth) * (Q_ALONG ? 1u : a.q_row) * 2;
    const uint64_t p_step = static_cast<uint64_t>(kGatedDepth) * (P_ALONG ? 1u : a.p_row) * 2;
    uint32_t ahead = s_begin, left = 0;     // its number, and the k from its first on
    const uint8_t *q_at = nullptr, *p_at = nullptr, *p_other = nullptr;
    auto seek = [&](uint32_t s) {
        const bool second = FORM == kInputGrad ? s >= half_steps : half != 0;
        const uint32_t in_half = FORM == kInputGrad && second ? s - half_steps : s;
        q_at = (second ? q_base[1] : q_base[0]) + in_half * q_step - kGatedBias;
        p_at = (second ? p_base[1] : p_base[0]) + in_half * p_step - kGatedBias;
        if constexpr (FORM == kForward)
            p_other = p_base[1] + in_half * p_step - kGatedBias;
        left = a.depth - in_half * kGatedDepth;
    };
    auto request_q = [&](auto ragged, auto number, uint32_t place) {
        q.template request<decltype(ragged)::value, decltype(number)::value>(q_at, lds_at + place, wave, left);
    };
    auto request_p = [&](auto ragged, auto number, uint32_t place) {
        constexpr bool RAGGED = decltype(ragged)::value;
        constexpr uint32_t N = decltype(number)::value;
        if constexpr (FORM != kForward)
            p.template request<RAGGED, N>(p_at, lds_at + place, wave, left);
        else if constexpr (N < Half::kCopies)
            half_p.template request<RAGGED, N>(p_at, lds_at + place, wave, left);
        else
            half_p.template request<RAGGED, N - Half::kCopies>(p_other, lds_at + place + Half::kBytes, wave, left);
    };
    auto advance = [&]() {
        ++ahead;
        q_at += q_step;
        p_at += p_step;
        if constexpr (FORM == kForward)
            p_other += p_step;
        left -= kGatedDepth;
        if constexpr (FORM == kInputGrad)
            if (ahead == half_steps)
                seek(ahead);
    };
    auto request_all = [&](uint32_t q_place, uint32_t p_place) {
        auto all_of = [&](auto ragged) {
            each_of<Q::kCopies>([&](auto n) { request_q(ragged, n, q_place); });
            each_of<P::kCopies>([&](auto n) { request_p(ragged, n, p_place); });
        };
        if (left >= kGatedDepth)
            all_of(std::false_type{});
        else
            all_of(std::true_type{});
        advance();
    };
    constexpr uint32_t kCopies = Q::kCopies + P::kCopies;

    // ---- what this wave multiplies
    const uint32_t wi = wave % 2, wj = wave / 2;
    const uint32_t q_lane = Q::lane_address(wi * (SIZE / 2), lane);
    const uint32_t p_lane = P::lane_address(FORM == kForward ? wj * (SIZE / 4) : wj * (SIZE / 2), lane);
    gated_f32x4_t acc[TILES][TILES];  // [j][i]
#pragma unroll
    for (int jt = 0; jt < TILES; ++jt)
#pragma unroll
        for (int it = 0; it < TILES; ++it)
            acc[jt][it] = gated_f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    // The operands of half a step are read into registers while the half before it is multiplied.  Once everyone has read a step's
    // second half, its places in LDS are free: during its second half the q of the step after the next (RING 2) is requested, during the first
    // half of the next step its p, which has a place more for that.  A CU takes in 64 bytes a cycle, half of a tile of 256's cycles of
    // products and all of one of 128's, so the requests are spread over both halves (all in one: input gradient of 2048 tokens without
    // slices 620 us, 575 so; in tiles of 128, 64 tokens, 252 / 204).
    struct Operands {
        gated_bf16x8_t q[TILES], p[TILES];
    };
    auto read_q = [&](Operands &o, uint32_t place, int n, uint32_t h) { o.q[n] = Q::read(lds + place, q_lane, n, h); };
    auto read_p = [&](Operands &o, uint32_t place, int n, uint32_t h) {
        // (kForward: the second half of the sums are the other weight's)
        if constexpr (FORM == kForward)
            o.p[n] = P::read(lds + place + (n >= TILES / 2 ? Half::kBytes : 0), p_lane, n % (TILES / 2), h);
        else
            o.p[n] = P::read(lds + place, p_lane, n, h);
    };
    static_assert(Q::kCopies == TILES && P::kCopies == TILES, "a copy to a row of sums");
    // how many of the copies requested last may still travel when the next step is read
    constexpr uint32_t kLater = (kQRing - 2) * kCopies + P::kCopies;
    constexpr uint32_t kOthers = (kQRing - 1) * kCopies;  // (the first step)
    static_assert(kLater < 64 && kOthers < 64, "as many as the counter counts");
    // (what is not a product stands by itself between products, in their shadow)
    auto row_of_sums = [&](auto requests, auto number, const Operands &now, Operands &then, uint32_t q_place, uint32_t p_place, auto h,
                           uint32_t to) {
        constexpr int n = decltype(number)::value, kEach = TILES / 4;
        auto some = [&](int from) {
#pragma unroll
            for (int it = from * kEach; it < (from + 1) * kEach; ++it)
                acc[n][it] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(now.p[n], now.q[it], acc[n][it], 0, 0, 0);
        };
        some(0);
        read_q(then, q_place, n, h);
        __builtin_amdgcn_sched_barrier(0);
        some(1);
        read_p(then, p_place, n, h);
        __builtin_amdgcn_sched_barrier(0);
        some(2);
        if constexpr (decltype(requests)::value && h == 1)
            request_p(std::false_type{}, number, to);
        else if constexpr (decltype(requests)::value)
            request_q(std::false_type{}, number, to);
        __builtin_amdgcn_sched_barrier(0);
        some(3);
        __builtin_amdgcn_sched_barrier(0);
    };
    // h: the half that is read meanwhile
    auto half_step = [&](auto requests, const Operands &now, Operands &then, uint32_t q_place, uint32_t p_place, auto h, uint32_t to) {
        each_of<TILES>([&](auto n) { row_of_sums(requests, n, now, then, q_place, p_place, h, to); });
    };
    if (steps > 0) {
        constexpr std::integral_constant<uint32_t, 0> kFirstHalf{};
        constexpr std::integral_constant<uint32_t, 1> kSecondHalf{};
        Operands first, second;
        uint32_t q_now = 0, p_now = kQEnd, p_before = kPEnd - P::kBytes;  // the step's places, and the one's before
        auto after = [](uint32_t place, uint32_t bytes, uint32_t begin, uint32_t end) { return place + bytes == end ? begin : place + bytes; };
        seek(s_begin);
        for (uint32_t r = 0; r < kQRing && r < steps; ++r)
            request_all(r * Q::kBytes, kQEnd + r * P::kBytes);
        if (steps >= kQRing)
            gated_arrive<kOthers>(lds);
        else
            gated_arrive<0>(lds);
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            read_q(first, 0, n, 0);
            read_p(first, kQEnd, n, 0);
        }
        for (uint32_t s = 0; s < steps;) {
            while (s + kQRing < steps && left >= kGatedDepth) {
                const uint32_t q_next = after(q_now, Q::kBytes, 0, kQEnd), p_next = after(p_now, P::kBytes, kQEnd, kPEnd);
                half_step(std::true_type{}, first, second, q_now, p_now, kSecondHalf, p_before);
                gated_arrive<kLater>(lds);
                half_step(std::true_type{}, second, first, q_next, p_next, kFirstHalf, q_now);
                advance();
                q_now = q_next;
                p_before = p_now;
                p_now = p_next;
                ++s;
            }
            // one by one: the last, and where half a sum ends
            const uint32_t q_next = after(q_now, Q::kBytes, 0, kQEnd), p_next = after(p_now, P::kBytes, kQEnd, kPEnd);
            half_step(std::false_type{}, first, second, q_now, p_now, kSecondHalf, 0);
            gated_arrive<0>(lds);
            if (s + kQRing < steps)
                request_all(q_now, p_before);
            half_step(std::false_type{}, second, first, q_next, p_next, kFirstHalf, 0);  // (behind the last step: what nobody uses)
            q_now = q_next;
            p_before = p_now;
            p_now = p_next;
            ++s;
        }
    }

    // ---- A lane holds, of every 16 x 16 sums, i = lane % 16 and four neighbouring j from 4 * (lane / 16) on.  Of four such
    // (two by two), rounded, the rows of 16 lanes trade pieces until a lane holds eight neighbouring j and a wave's store 64 bytes
    // each of 16 rows: 8 bytes to a lane, as they come, were 32 bytes each, and twice the stores.
    constexpr int kOutputs = FORM == kForward ? TILES / 2 : TILES;  // tiles of j
    const uint32_t j_lane = j0 + wj * (kOutputs * 16) + lane / 16 % 2 * 16 + lane / 32 * 8;
    const uint32_t i_lane = i0 + wi * (SIZE / 2) + lane % 16;
    auto leave = [&](uint16_t *c, int jt, int it, auto words) {
        uint32_t v[2][4];  // [jt, jt + 1]
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const auto r = __builtin_amdgcn_permlane16_swap(words(jt + t, it, e), words(jt + t, it + 1, e), false, false);
                v[t][e] = r[0];
                v[t][2 + e] = r[1];
            }
        uint32_t at[2][4];  // [it, it + 1]
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            const auto r = __builtin_amdgcn_permlane16_swap(v[0][d], v[1][d], false, false);
            at[0][d] = r[0];
            at[1][d] = r[1];
        }
        const uint32_t j = j_lane + jt * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t i = i_lane + (it + t) * 16;
            if (i < a.rows && j < a.cols)
                *reinterpret_cast<uint4 *>(c + static_cast<uint64_t>(i) * a.c_row + j) = make_uint4(at[t][0], at[t][1], at[t][2], at[t][3]);
        }
    };
    // (in binary32 four neighbouring j are 16 bytes, and a wave's store 64 of each row as it is)
    auto leave_sum = [&](float *c, const gated_f32x4_t &v, int jt, int it) {
        const uint32_t i = i_lane + it * 16, j = j0 + wj * (kOutputs * 16) + jt * 16 + lane / 16 * 4;
        if (i < a.rows && j < a.cols)
            *reinterpret_cast<float4 *>(c + static_cast<uint64_t>(i) * a.c_row + j) = make_float4(v[0], v[1], v[2], v[3]);
    };
    if (FORM == kInputGrad && a.partial) {
        float *c = a.partial + static_cast<uint64_t>(slice) * a.rows * a.c_row;
#pragma unroll
        for (int jt = 0; jt < TILES; ++jt)
#pragma unroll
            for (int it = 0; it < TILES; ++it) {
                asm volatile("" : "+a"(acc[jt][it]));  // (see below)
                leave_sum(c, acc[jt][it], jt, it);
            }
        return;
    }
#pragma unroll
    for (int jt = 0; jt < kOutputs; jt += 2) {
#pragma unroll
        for (int it = 0; it < TILES; it += 2) {
            // (a group's sums leave the accumulation registers when it is their turn, not all at once)
#pragma unroll
            for (int t = 0; t < (FORM == kForward ? 8 : 4); ++t)
                asm volatile("" : "+a"(acc[jt + t % 2 + t / 4 * (TILES / 2)][it + t / 2 % 2]));
            auto sums = [&](int j, int i, int e) { return pack_bf16(acc[j][i][2 * e], acc[j][i][2 * e + 1]); };
            if constexpr (FORM == kForward) {
                auto products = [&](int j, int i, int e) {
                    const gated_f32x4_t &g = acc[j][i], &u = acc[j + TILES / 2][i];
                    return pack_bf16(gated_value(g[2 * e], a.activation) * u[2 * e], gated_value(g[2 * e + 1], a.activation) * u[2 * e + 1]);
                };
                leave(a.c[0], jt, it, products);
                if (a.gate) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        leave_sum(a.gate, acc[jt + t % 2][it + t / 2], jt + t % 2, it + t / 2);
                        leave_sum(a.up, acc[jt + t % 2 + TILES / 2][it + t / 2], jt + t % 2, it + t / 2);
                    }
                }
            } else {
                leave(half ? a.c[1] : a.c[0], jt, it, sums);
            }
        }
    }
}

template <GatedForm FORM, int SIZE, int RING>
__global__ __launch_bounds__(kGatedThreads, SIZE == 128 && RING == 2 ? 2 : 1) void gated_kernel(const GatedArgs a)
{
    gated_workgroup<FORM, SIZE, RING>(a, blockIdx.x, gridDim.x);
}

// The input gradient and the weight gradients in one launch.
__global__ __launch_bounds__(kGatedThreads, 2) void gated_gradients_kernel(const GatedArgs x, const GatedArgs w, const uint32_t x_wgs)
{
    if (blockIdx.x < x_wgs)
        gated_workgroup<kInputGrad, 128, 2>(x, blockIdx.x, x_wgs);
    else
        gated_workgroup<kWeightGrad, 128, 2>(w, blockIdx.x - x_wgs, gridDim.x - x_wgs);
}

// dg = dh * u * act'(g), du = dh * act(g), each rounded to bf16 once (the matrix cores take bf16; with g and u rounded before, the
// gradients were off by 3.1e-3 in the mean, 2.3e-3 now, of which the roundings of the results are 1.7e-3), 8 elements to a thread.
// act'(g) = s + g s (1 - s) z'(g), s = sigmoid(z(g)); z' of the GELU grows with g^2, where s (1 - s) has long been zero.
// Bound by memory: 14 bytes an element, 2048 x 14336 in 77 us = 5.3 TB/s.
constexpr uint32_t kGatedSlopeThreads = 256;
__global__ __launch_bounds__(kGatedSlopeThreads) void gated_slope_kernel(const float4 *__restrict__ gate, const float4 *__restrict__ up,
                                                                         const uint4 *__restrict__ grad_h, uint4 *__restrict__ dg,
                                                                         uint4 *__restrict__ du, uint64_t pieces, uint32_t activation)
{
    const uint64_t at = static_cast<uint64_t>(blockIdx.x) * kGatedSlopeThreads + threadIdx.x;
    if (at >= pieces)
        return;
    const float4 g0 = gate[2 * at], g1 = gate[2 * at + 1], u0 = up[2 * at], u1 = up[2 * at + 1];
    const uint4 h4 = grad_h[at];
    const float gs[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w}, us[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
    const uint32_t hs[4] = {h4.x, h4.y, h4.z, h4.w};
    uint32_t dgs[4], dus[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float dgv[2], duv[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float g = gs[2 * i + e], u = us[2 * i + e];
            const float h = __uint_as_float(e ? hs[i] & 0xFFFF0000u : hs[i] << 16);
            const float s = gated_sigmoid(gated_argument(g, activation));
            const float slope = activation ? kGeluScale * (1.0f + 0.134145f * fminf(g * g, 1e4f)) : 1.0f;
            dgv[e] = h * u * (s + g * (s * (1.0f - s)) * slope);
            duv[e] = h * (g * s);
        }
        dgs[i] = pack_bf16(dgv[0], dgv[1]);
        dus[i] = pack_bf16(duv[0], duv[1]);
    }
    dg[at] = make_uint4(dgs[0], dgs[1], dgs[2], dgs[3]);
    du[at] = make_uint4(dus[0], dus[1], dus[2], dus[3]);
}

// dx from the sums of the slices of k, in their order, 8 elements to a thread.  Bound by memory: two slices of 2048 x 4096 12.7 us = 6.6 TB/s.
__global__ __launch_bounds__(kGatedSlopeThreads) void gated_join_kernel(const float4 *__restrict__ partial, uint4 *__restrict__ out,
                                                                        uint64_t pieces, uint32_t slices)
{
    const uint64_t at = static_cast<uint64_t>(blockIdx.x) * kGatedSlopeThreads + threadIdx.x;
    if (at >= pieces)
        return;
    float4 a = partial[2 * at], b = partial[2 * at + 1];
    for (uint32_t s = 1; s < slices; ++s) {
        const float4 c = partial[2 * (s * pieces + at)], d = partial[2 * (s * pieces + at) + 1];
        a.x += c.x;
        a.y += c.y;
        a.z += c.z;
        a.w += c.w;
        b.x += d.x;
        b.y += d.y;
        b.z += d.z;
        b.w += d.w;
    }
    out[at] = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
}

// h from the two sums in binary32, as the compressed weights' product leaves them (serving), four to a thread.
__global__ __launch_bounds__(kGatedSlopeThreads) void gated_product_kernel(const float *__restrict__ gate, const float *__restrict__ up,
                                                                           uint16_t *__restrict__ h, uint64_t count, uint32_t activation)
{
    const uint64_t at = (static_cast<uint64_t>(blockIdx.x) * kGatedSlopeThreads + threadIdx.x) * 4;
    if (at + 4 <= count && (reinterpret_cast<uintptr_t>(h) & 7u) == 0) {
        const float4 g = *reinterpret_cast<const float4 *>(gate + at), u = *reinterpret_cast<const float4 *>(up + at);
        *reinterpret_cast<uint2 *>(h + at) = make_uint2(pack_bf16(gated_value(g.x, activation) * u.x, gated_value(g.y, activation) * u.y),
                                                        pack_bf16(gated_value(g.z, activation) * u.z, gated_value(g.w, activation) * u.w));
        return;
    }
    for (uint64_t i = at; i < at + 4 && i < count; ++i)
        h[i] = static_cast<uint16_t>(pack_bf16(gated_value(gate[i], activation) * up[i], 0.0f));
}

}  // namespace nz
