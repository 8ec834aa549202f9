// The ragged sequences of a call on the cache (neuzip_sequences.h), on the host: every token of every sequence is in one tile, whatever the tensors
// say no row, page or table entry is out of range.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <utility>
#include <vector>

#include "neuzip_sequences.h"

using namespace nz;

static void require(bool ok, const char *what)
{
    if (!ok) {
        std::printf("%s\n", what);
        std::exit(1);
    }
}

// the last s with first_tile(s) <= id
static uint32_t sequence_of(const std::vector<int32_t> &starts, uint32_t count, const TileNumbers &t, uint64_t id)
{
    uint32_t found = count;
    for (uint32_t s = 0; s < count; ++s)
        if (first_tile(t, starts[s], s) <= id)
            found = s;
    return found;
}

int main()
{
    std::mt19937 random(7);
    const auto below = [&](uint32_t n) { return static_cast<int32_t>(random() % n); };
    for (int turn = 0; turn < 4000; ++turn) {
        const bool broken = turn % 4 == 3;  // whatever the tensors say
        const uint32_t count = 1 + below(9), shift = 4 + below(4), width = 1 + below(5), pages = 1 + below(30);
        const uint32_t page = 1u << shift;
        std::vector<int32_t> starts(count + 1), lengths(count), table(count * width);
        starts[0] = below(3) ? 0 : below(5);
        for (uint32_t s = 0; s < count; ++s) {
            const int32_t room = static_cast<int32_t>(width * page);
            lengths[s] = below(4) ? 1 + below(room) : below(room + 40);
            const int32_t rows = below(3) ? below(lengths[s] + 1) : below(4);
            starts[s + 1] = starts[s] + rows;
            for (uint32_t i = 0; i < width; ++i)
                table[s * width + i] = below(8) ? below(pages) : below(3) - 1 + below(2) * 1000000;
        }
        uint32_t rows = starts[count] + below(4);
        if (broken) {
            for (int i = 0; i < 3; ++i) {
                const int32_t odd[] = {-1, -2147483647 - 1, 2147483647, below(1000), 0};
                starts[below(count + 1)] = odd[below(5)];
                lengths[below(count)] = odd[below(5)];
            }
            rows = below(300);
        }
        const SequencesView v = {starts.data(), lengths.data(), table.data(), count, width, rows, shift, pages};
        for (uint32_t s = 0; s < count; ++s) {
            const NewTokens n = new_tokens(v, s);
            require(n.begin + static_cast<uint64_t>(n.count) <= rows, "rows");
            require(n.length <= width * page && (n.length == 0 || (n.count <= n.length && n.first == n.length - n.count)), "positions");
            if (!broken)
                require(n.count == static_cast<uint32_t>(starts[s + 1] - starts[s]) &&
                        (n.count == 0 || (n.length != 0) == (lengths[s] >= static_cast<int32_t>(n.count) && lengths[s] <= static_cast<int32_t>(width * page))), "tokens");
            for (uint32_t number = 0; number < width + 3; ++number) {
                const uint32_t p = page_of(v, s, number);
                require(p == kNoPage || (p < pages && number < width && table[s * width + number] == static_cast<int32_t>(p)), "page");
                if (number < width && table[s * width + number] >= 0 && table[s * width + number] < static_cast<int32_t>(pages))
                    require(p != kNoPage, "a page that is there");
            }
        }
        if (broken)
            continue;
        // pages that tokens go to
        {
            const TileNumbers t = {shift, 1, 2};
            std::map<std::pair<uint32_t, uint32_t>, int> got;
            for (uint64_t id = 0; id < tile_count(t, rows, count); ++id) {
                const uint32_t s = sequence_of(starts, count, t, id);
                if (s >= count)
                    continue;
                const NewTokens n = new_tokens(v, s);
                const uint32_t number = (n.first >> shift) + static_cast<uint32_t>(id - first_tile(t, starts[s], s));
                if (n.length == 0 || number > (n.length - 1) >> shift)
                    continue;
                ++got[{s, number}];
            }
            size_t want = 0;
            for (uint32_t s = 0; s < count; ++s) {
                const NewTokens n = new_tokens(v, s);
                if (n.length)
                    for (uint32_t number = n.first >> shift; number <= (n.length - 1) >> shift; ++number, ++want)
                        require(got[{s, number}] == 1, "a page once");
            }
            require(got.size() == want, "no other pages");
        }
        // tiles of rows
        for (uint32_t tile_shift : {0u, 4u, 5u, 7u}) {
            const uint32_t unit = 1u << tile_shift, group = unit == 1 ? 1 : 1 + below(9);
            const TileNumbers t = {tile_shift, group, unit == 1 ? 0u : 1u};
            std::map<std::pair<uint32_t, uint32_t>, int> got;
            for (uint64_t id = 0; id < tile_count(t, rows, count); ++id) {
                const uint32_t s = sequence_of(starts, count, t, id);
                if (s >= count)
                    continue;
                const NewTokens n = new_tokens(v, s);
                const uint64_t row0 = (id - first_tile(t, starts[s], s)) * unit;
                for (uint64_t r = row0; r < row0 + unit && r < static_cast<uint64_t>(n.count) * group; ++r)
                    ++got[{s, static_cast<uint32_t>(r)}];
            }
            size_t want = 0;
            for (uint32_t s = 0; s < count; ++s)
                for (uint32_t r = 0; r < new_tokens(v, s).count * group; ++r, ++want)
                    require(got[{s, r}] == 1, "a row once");
            require(got.size() == want, "no other rows");
        }
        // tiles of rows that are counted row by row
        for (uint32_t unit : {16u, 32u, 128u}) {
            const uint32_t group = 1 + below(40);
            const TileNumbers t = {0, (group + unit - 1) / unit, 0};
            std::map<std::pair<uint32_t, uint32_t>, int> got;
            for (uint64_t id = 0; id < tile_count(t, rows, count); ++id) {
                const uint32_t s = sequence_of(starts, count, t, id);
                if (s >= count)
                    continue;
                const NewTokens n = new_tokens(v, s);
                const uint64_t row0 = (id - first_tile(t, starts[s], s)) * unit;
                for (uint64_t r = row0; r < row0 + unit && r < static_cast<uint64_t>(n.count) * group; ++r)
                    ++got[{s, static_cast<uint32_t>(r)}];
            }
            size_t want = 0;
            for (uint32_t s = 0; s < count; ++s)
                for (uint32_t r = 0; r < new_tokens(v, s).count * group; ++r, ++want)
                    require(got[{s, r}] == 1, "a row once, counted by rows");
            require(got.size() == want, "no other rows, counted by rows");
        }
    }
    std::printf("ok\n");
    return 0;
}
