// The rules of the 8-bit expert FFN (spice_internal.h) on calls read from stdin, one per line as
// "T d N K C I Is": prints the tile shape, the parts of the shared block's down contraction, whether an
// XCD takes neighbouring tiles, the bytes of the parts' sums, and the shape's rows and tokens.
#include <cstdio>

#include "spice_internal.h"

int main() {
    int T, d, N, K, C, I, Is;
    while (std::scanf("%d %d %d %d %d %d %d", &T, &d, &N, &K, &C, &I, &Is) == 7) {
        const spice::I8Plan p = spice::i8_plan(T, d, N, K, C, I, Is);
        std::printf("%d %d %d %zu %d %d\n", p.shape, p.parts, p.xcd, spice::i8_part_bytes(p, T, d),
                    spice::kI8Shapes[p.shape].rows, spice::kI8Shapes[p.shape].tokens);
    }
}
