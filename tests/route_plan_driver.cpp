// The rule of the scored routing (spice_internal.h) on calls read from stdin, one per line as
// "T N d dtype part_bytes x_to_host": prints whether it keeps the rows, the contraction's parts, the chunks
// that a group's blocks share the experts in, and the experts of a chunk.
#include <cstdio>

#include "spice_internal.h"

int main() {
    int T, N, d, dtype, host;
    long long bytes;
    while (std::scanf("%d %d %d %d %lld %d", &T, &N, &d, &dtype, &bytes, &host) == 6) {
        const spice::ScoredPlan p = spice::scored_plan(T, N, d, dtype, (size_t)bytes, host != 0);
        std::printf("%d %d %d %d\n", p.rows, p.parts, p.chunks, p.chunk);
    }
}
