// The cut of the selective scan (csrc/la_scan_cut.h) on its own: reads sizes from stdin, prints how sequences are cut.
//   in   B N E G S
//   out  tiles pieces piece_tiles (forwards)  tiles pieces piece_tiles (backwards)
#include <cstdio>

#include "../paper_2006_16236_amd/csrc/la_scan_cut.h"

int main() {
    int B, N, E, G, S;
    while (std::scanf("%d %d %d %d %d", &B, &N, &E, &G, &S) == 5) {
        for (int backward = 0; backward < 2; ++backward) {
            const la::ScanCut c = la::scan_cut_of(B, N, E, G, S, backward != 0);
            std::printf("%d %d %d%c", c.tiles, c.pieces, c.piece_tiles, backward ? '\n' : ' ');
        }
    }
    return 0;
}
