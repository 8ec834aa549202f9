// The ragged sequences of a call on the cache: which rows are whose, and where a position's page is.  What the caller's tensors say is checked
// here, element by element, so that no kernel leaves its buffers whatever they hold.  (No device code in here: a host program can include it.)
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define NZ_BOTH __host__ __device__ __forceinline__
#else
#define NZ_BOTH inline
#endif

namespace nz {

struct SequencesView {
    const int32_t *starts, *lengths, *table;
    uint32_t count, table_width;
    uint32_t rows;        // of the call's tensors
    uint32_t page_shift;  // page_tokens = 1 << page_shift
    uint32_t pages;       // of the cache
};

// The newest tokens of one sequence.
struct NewTokens {
    uint32_t begin, count;  // rows
    uint32_t first;         // the position of the first of them
    uint32_t length;        // of the sequence, with them; 0: it is left out
};

// begin, end, length: starts[s], starts[s + 1] and lengths[s]
NZ_BOTH NewTokens new_tokens(const SequencesView &v, int32_t begin, int32_t end, int32_t length)
{
    NewTokens t = {0, 0, 0, 0};
    if (begin < 0 || end <= begin || static_cast<uint32_t>(end) > v.rows)
        return t;
    t.begin = static_cast<uint32_t>(begin);
    t.count = static_cast<uint32_t>(end - begin);
    if (length < end - begin || static_cast<uint64_t>(length) > (static_cast<uint64_t>(v.table_width) << v.page_shift))
        return t;
    t.length = static_cast<uint32_t>(length);
    t.first = t.length - t.count;
    return t;
}
NZ_BOTH NewTokens new_tokens(const SequencesView &v, uint32_t s) { return new_tokens(v, v.starts[s], v.starts[s + 1], v.lengths[s]); }

constexpr uint32_t kNoPage = 0xFFFFFFFFu;

// The page of number `number` of sequence s.
NZ_BOTH uint32_t page_of(const SequencesView &v, uint32_t s, uint32_t number)
{
    if (number >= v.table_width)
        return kNoPage;
    const int32_t page = v.table[static_cast<uint64_t>(s) * v.table_width + number];
    return page >= 0 && static_cast<uint32_t>(page) < v.pages ? static_cast<uint32_t>(page) : kNoPage;
}

// A call's work is cut into tiles that lie in one sequence each, up to 2^shift rows (or rows times `group`) long; how many a sequence has is known
// on the device alone.  So each sequence gets a range of numbers that is sure to be long enough, from where the rows before it would end if they
// lay in whole tiles, and `slack` more for each sequence; numbers that no tile takes have nothing to do.  With u = 2^shift:
//   n rows in tiles of their own: ceil(n / u) <= floor((a + n) / u) - floor(a / u) + 1, slack 1
//   n tokens in pages of u, from anywhere in a page on: ceil(n / u) + 1 at most, slack 2
//   a row's own number, or `group` of them (shift 0): slack 0
struct TileNumbers {
    uint32_t shift, group, slack;
};
NZ_BOTH uint64_t first_tile(const TileNumbers &t, int32_t start, uint32_t s)
{
    return (start > 0 ? static_cast<uint64_t>(start) * t.group >> t.shift : 0) + static_cast<uint64_t>(t.slack) * s;
}
NZ_BOTH uint64_t tile_count(const TileNumbers &t, uint32_t rows, uint32_t count)
{
    return (static_cast<uint64_t>(rows) * t.group >> t.shift) + static_cast<uint64_t>(t.slack) * count;
}

}  // namespace nz
