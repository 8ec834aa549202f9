// What the library's rule says of calls of the attention: a line of heads, head_dim, page, sequences, query heads, rows, window and longest each in, rows and waves to a
// workgroup and splits out.
#include <cstdio>

#include "neuzip_attention_shape.h"

int main()
{
    unsigned heads, dim, page, count, q_heads, rows, window;
    unsigned long long longest;
    while (std::scanf("%u %u %u %u %u %u %u %llu", &heads, &dim, &page, &count, &q_heads, &rows, &window, &longest) == 8) {
        const nz::AttendShape s = nz::attend_shape(heads, dim, page, count, q_heads, rows, window, longest);
        std::printf("%u %u %u\n", s.rows, s.waves, s.splits);
    }
    return 0;
}
