// Prints the forms that calls of the gated block take: a line of "tokens in_features out_features" in, one of
// "forward size, ring; input gradient size, ring, slices; weight gradients size, ring; slices of both in one launch (0: apart)" out.
#include <cstdio>

#include "neuzip_gated_shape.h"

int main()
{
    unsigned long long tokens, in, out;
    while (std::scanf("%llu %llu %llu", &tokens, &in, &out) == 3) {
        const nz::GatedShape f = nz::gated_shape<nz::kForward>(tokens, out, in), x = nz::gated_shape<nz::kInputGrad>(tokens, in, out),
                             w = nz::gated_shape<nz::kWeightGrad>(out, in, tokens);
        std::printf("%u %u %u %u %u %u %u %u\n", f.size, f.ring, x.size, x.ring, x.slices, w.size, w.ring, nz::gated_beside(tokens, out, in));
    }
    return 0;
}
