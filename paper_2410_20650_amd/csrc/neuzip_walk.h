// What the kernels that walk rANS states share: one decoding step, the merging of decoded exponents with their fields, the slot
// table, and scans over the lanes of a wave.
#pragma once

#include "neuzip_format.h"

namespace nz {

// binary32 -> bf16, round to nearest even: the conversion instruction of gfx950
__device__ __forceinline__ uint32_t bf16_of(float v)
{
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

__device__ __forceinline__ bool bf16_is_nan(uint32_t u) { return (u & 0x7FFFu) > 0x7F80u; }

__device__ __forceinline__ uint32_t normalise_word(uint32_t u, float c)
{
    if (bf16_is_nan(u))
        return u | 0x40u;
    return bf16_of(__uint_as_float(u << 16) / c);
}

__device__ __forceinline__ float coefficient(uint32_t coef) { return 1.0f + static_cast<float>(coef) * 0.0078125f; }

// Stores and atomics issued so far by this wave have been performed (their acknowledgements are in)
// before anything that follows.
__device__ __forceinline__ void wait_for_memory_acks() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Inclusive scan of v over the 64 lanes of the wave with data-parallel-primitive moves (vector ALU
// rate: no trip through the LDS crossbar as with a lane shuffle): inside each row of 16 lanes by
// shifts of 1, 2, 4, 8 (a lane without a source keeps the identity), then the last lane of rows 0
// and 2 is added into rows 1 and 3, then lane 31 into rows 2 and 3.  All 64 lanes must be active.
template <class Op>
__device__ __forceinline__ uint32_t row_scan_u32(uint32_t v, uint32_t identity, Op op)
{
#define NZ_DPP(ctrl, rows) \
    static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(identity), static_cast<int>(v), ctrl, rows, 0xf, false))
    v = op(v, NZ_DPP(0x111, 0xf));  // row_shr:1
    v = op(v, NZ_DPP(0x112, 0xf));  // row_shr:2
    v = op(v, NZ_DPP(0x114, 0xf));  // row_shr:4
    v = op(v, NZ_DPP(0x118, 0xf));  // row_shr:8
    return v;
}

template <class Op>
__device__ __forceinline__ uint32_t wave_scan_u32(uint32_t v, uint32_t identity, Op op)
{
    v = row_scan_u32(v, identity, op);
    v = op(v, NZ_DPP(0x142, 0xa));  // row_bcast:15 into rows 1 and 3
    v = op(v, NZ_DPP(0x143, 0xc));  // row_bcast:31 into rows 2 and 3
#undef NZ_DPP
    return v;
}

struct OpAdd {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a + b; }
};
struct OpMax {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};

// Inclusive sum over the lanes of a row of 16 (all of them active).
__device__ __forceinline__ uint32_t row_scan_u32(uint32_t v) { return row_scan_u32(v, 0u, OpAdd{}); }

// ... and of a half of 32.
__device__ __forceinline__ uint32_t half_scan_u32(uint32_t v)
{
    v = row_scan_u32(v);
    // row_bcast:15 into rows 1 and 3
    return v + static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x142, 0xa, 0xf, false));
}

// Sum / maximum over the wave, the same value in every lane (lane 63 of the scan, read out as a scalar).
__device__ __forceinline__ uint32_t wave_sum_u32(uint32_t v)
{
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(wave_scan_u32(v, 0u, OpAdd{})), 63));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(wave_scan_u32(v, 0u, OpMax{})), 63));
}

template <int KB>
__device__ __forceinline__ uint64_t load_fields(const uint8_t *__restrict__ sm, uint64_t first_elem)
{
    // the (KB+1)*8 field bits of 8 neighbouring elements
    if constexpr (KB == 7) {
        const uint2 v = *reinterpret_cast<const uint2 *>(sm + first_elem);
        return static_cast<uint64_t>(v.x) | (static_cast<uint64_t>(v.y) << 32);
    } else if constexpr (KB == 3) {
        return *reinterpret_cast<const uint32_t *>(sm + first_elem / 2);
    } else if constexpr (KB == 1) {
        return *reinterpret_cast<const uint16_t *>(sm + first_elem / 4);
    } else {
        return sm[first_elem / 8];
    }
}

// Two bf16 words (sign << 15 | exponent << 7 | kept mantissa bits << (7 - KB)) from the field
// bits of a pair of neighbouring elements and the two slot-table entries that decoded them
// (exponent in the low byte of an entry).
template <int KB>
__device__ __forceinline__ uint32_t merge_pair(uint64_t fields, int pair, uint32_t entry_lo, uint32_t entry_hi)
{
    // [0, exponent_hi, 0, exponent_lo]
    const uint32_t expo = __builtin_amdgcn_perm(entry_hi, entry_lo, 0x0c040c00u);
    if constexpr (KB == 7) {
        // lossless: a field is the byte sign << 7 | mantissa.  Spread the two bytes over the two
        // halfwords ([b1, b1, b0, b0]) and keep bit 15 and bits 6..0 of each.
        const uint32_t half = static_cast<uint32_t>(fields >> (32 * (pair >> 1)));
        const uint32_t twice = __builtin_amdgcn_perm(half, half, (pair & 1) ? 0x03030202u : 0x01010000u);
        return (expo << 7) | (twice & 0x807F807Fu);
    } else if constexpr (KB == 3) {
        // byte `pair` of the 32 field bits holds two nibbles s m2 m1 m0 (low nibble = first element).
        // Nibbles into halfwords, then one multiply by 2^4 + 2^12 puts m at bits 6..4 and s at bit 15.
        const uint32_t v = static_cast<uint32_t>(fields);
        const uint32_t even = v & 0x0F0F0F0Fu, odd = (v >> 4) & 0x0F0F0F0Fu;
        const uint32_t nib = __builtin_amdgcn_perm(odd, even, 0x0c000c00u | ((4u + pair) << 16) | pair);
        return (expo << 7) | (__umul24(nib, 0x1010u) & 0x80708070u);
    } else if constexpr (KB == 1) {
        // nibble `pair` of the 16 field bits is s1 m1 s0 m0: m0 -> bit 6, s0 -> 15, m1 -> 22, s1 -> 31
        const uint32_t f2 = (static_cast<uint32_t>(fields) >> (4 * pair)) & 0xFu;
        const uint32_t spread = __umul24(f2 << 16, 0x1010u) + __umul24(f2, 0x4040u);
        return (expo << 7) | (spread & 0x80408040u);
    } else {
        // bits 2*pair and 2*pair + 1 of the 8 field bits are the two signs
        const uint32_t v = static_cast<uint32_t>(fields);
        return (expo << 7) | ((v << (15 - 2 * pair)) & 0x8000u) | ((v << (30 - 2 * pair)) & 0x80000000u);
    }
}

struct LdsWords {
    const uint8_t *base;  // LDS copy of the workgroup's runs
    __device__ __forceinline__ uint32_t peek(uint32_t at) const { return *reinterpret_cast<const uint16_t *>(base + at); }
};
struct GlobalWords {
    const uint8_t *base;  // the lane's run inside the blob
    __device__ __forceinline__ uint32_t peek(uint32_t at) const { return *reinterpret_cast<const uint16_t *>(base + at); }
};
struct NoWords {
    __device__ __forceinline__ uint32_t peek(uint32_t) const { return 0; }
};

// One rANS decoding step of a lane's state; returns the slot-table entry (symbol in its low
// byte).  `next` always holds the word at byte position wp of the lane's word source, so a
// refill is a shift-or.
//   EAGER = false: the following word is fetched only where one has been consumed, behind a branch over the wave's mask.
//   EAGER = true: no branch; the refilled state is selected and the word at wp is fetched again whether it moved or not.
// A wave that has its SIMD to itself issues an instruction about every 8 cycles whatever it depends on, and the mask's
// save, branch and restore cost more there than the two selects: 116 cycles a symbol without them, 139 with (the loop alone,
// 1 to 4 waves per CU; at 8 waves 132 and 147).  With four waves per SIMD the vector unit's time counts, and the branch skips
// some of it: 30 M elements walked whole, k = 3, 26.3 us, without the branch 28.7.
template <bool EAGER, class WordSrc>
__device__ __forceinline__ uint32_t rans_get(const uint32_t *__restrict__ lut, uint32_t &x, uint32_t &wp,
                                             uint32_t &next, const WordSrc &src)
{
    const uint32_t e = lut[x & (kM - 1)];
    const uint32_t y = __umul24((e >> 8) & 0xFFFu, x >> kProbBits) + (e >> 20);
    if constexpr (EAGER) {
        const bool refill = y < kRansL;
        x = refill ? (y << 16) | next : y;
        wp = refill ? wp + 2 : wp;
        next = src.peek(wp);
    } else {
        x = y;
        if (x < kRansL) {
            x = (x << 16) | next;
            wp += 2;
            next = src.peek(wp);
        }
    }
    return e;
}

// bf16(stored * c) on the two halves of a merged dword: two multiplies, one packed conversion;
// a NaN keeps its bits and gets the quiet bit, as in normalise_word
__device__ __forceinline__ uint32_t denormalise_pair(uint32_t d, float c)
{
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2_t;
    typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2_t;
    const f32x2_t prod = {__fmul_rn(__uint_as_float(d << 16), c), __fmul_rn(__uint_as_float(d & 0xFFFF0000u), c)};
    uint32_t r = __builtin_bit_cast(uint32_t, __builtin_convertvector(prod, bf16x2_t));
    // c lies in [1, 2): a product is a NaN only if the stored word is one; one compare finds either
    if (__builtin_expect(__builtin_isunordered(prod[0], prod[1]), 0)) {
        if (bf16_is_nan(d & 0xFFFFu))
            r = (r & 0xFFFF0000u) | (d & 0xFFFFu) | 0x40u;
        if (bf16_is_nan(d >> 16))
            r = (r & 0x0000FFFFu) | (d & 0xFFFF0000u) | 0x400000u;
    }
    return r;
}

// 16 bytes per lane from memory straight into LDS: lane l's piece goes to `to` (the same for the wave) + 16 l.
__device__ __forceinline__ void copy_to_lds(const uint4 *from, uint8_t *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(from),
                                     (__attribute__((address_space(3))) void *)(to), 16, 0, 0);
}

// A barrier for what the workgroup's waves have written to LDS themselves, which does not wait for direct copies.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The slot table from the occupied symbols (TableBlock::steps, in LDS), by the whole workgroup; begins: the steps that pieces
// threadIdx.x and threadIdx.x + blockDim.x (of eight neighbouring slots) begin in.  First every piece is written as if the
// step it begins in filled it, then every step that starts inside a piece writes its slots of that piece over that: some 60
// instructions per thread of 256 and a barrier, while a search slot by slot (make_piece) takes 200 for each of its two pieces,
// and these tables are made by waves that wait for nothing else.  (The caller's barrier is still to come.)
__device__ __forceinline__ void make_table(const uint32_t *__restrict__ steps, const uint32_t (&begins)[2],
                                           const TableBlock *__restrict__ tb, uint32_t *__restrict__ lut)
{
    const uint32_t tid = threadIdx.x, threads = blockDim.x;
    auto entry = [](uint32_t here, uint32_t there, uint32_t slot) {
        return (here & 0xFFu) | ((((there >> 8) - (here >> 8)) & 0xFFFu) << 8) | ((slot - (here >> 8)) << 20);
    };
    auto fill = [&](uint32_t piece, uint32_t r) {
        const uint32_t e = entry(steps[r], steps[r + 1], piece * 8);
        uint4 *at = reinterpret_cast<uint4 *>(lut) + 2 * piece;
        at[0] = make_uint4(e, e + (1u << 20), e + (2u << 20), e + (3u << 20));
        at[1] = make_uint4(e + (4u << 20), e + (5u << 20), e + (6u << 20), e + (7u << 20));
    };
#pragma unroll
    for (uint32_t r = 0; r < 2; ++r)
        if (tid + r * threads < kM / 8)
            fill(tid + r * threads, begins[r]);
    for (uint32_t piece = tid + 2 * threads; piece < kM / 8; piece += threads)  // (small workgroups)
        fill(piece, tb->step_of[piece]);
    lds_barrier();
    for (uint32_t i = tid; i + 1 < kSteps; i += threads) {
        const uint32_t here = steps[i], there = steps[i + 1];
        const uint32_t from = here >> 8, piece_end = (from + 7) & ~7u;  // (nothing to write where a piece begins with it)
        const uint32_t upto = (there >> 8) < piece_end ? there >> 8 : piece_end;
        for (uint32_t slot = from; slot < upto; ++slot)
            lut[slot] = entry(here, there, slot);
    }
}

}  // namespace nz
