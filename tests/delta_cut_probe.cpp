// The cut of the gated delta rule (csrc/la_delta_cut.h) on its own: reads sizes from stdin, prints how sequences are cut.
//   in   heads D M chunks bytes
//   out  pieces length
#include <cstdio>

#include "../paper_2006_16236_amd/csrc/la_delta_cut.h"

int main() {
    long heads;
    int D, M, chunks, bytes;
    while (std::scanf("%ld %d %d %d %d", &heads, &D, &M, &chunks, &bytes) == 5) {
        const la::DeltaCut c = la::delta_cut_of(heads, D, M, chunks, bytes);
        std::printf("%d %d\n", c.pieces, c.length);
    }
    return 0;
}
