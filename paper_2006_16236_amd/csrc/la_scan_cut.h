// How the selective scan cuts its sequences into pieces (host code, without a GPU's headers).
#pragma once

namespace la {

// The scan's tokens go in tiles of kScanTile; the states before each tile are what a backward starts from.
constexpr int kScanTile = 16, kScanLanes = 64;                    // tokens of a tile, channels of a workgroup

// channel blocks of all groups
inline int scan_blocks(int E, int G) { return G * ((E / G + kScanLanes - 1) / kScanLanes); }

namespace scan_cost {
// Microseconds a tile of 16 tokens takes while every compute unit has 1, 2, .. `most` workgroups (its LDS holds no more),
// and what each 256 workgroups of the kernel that only forms the pieces' states add; measured with 2048 channels, bf16.
struct TileCost {
    int most;
    double us[3], local;
};
constexpr int kUnits = 256;
// Sixteen states: eight waves of two states while a compute unit has one workgroup, else four waves of four (1.95 us
// alone, but up to three fit: 3.6 us for the three, and 4.4 for three of the others, one after the other).  32 states: eight
// waves of four (2.5 us), else four of eight (2.7 alone, 4.1 for the two that fit; of the others 4.9).
inline TileCost fwd(int S) {
    return S == 8 ? TileCost{3, {1.53, 2.0, 2.6}, 0.6} : S == 16 ? TileCost{3, {1.47, 2.7, 3.6}, 0.9} : TileCost{2, {2.5, 4.1}, 1.6};
}
inline TileCost bwd(int S) {
    return S == 8 ? TileCost{2, {3.3, 4.8}, 0.6} : S == 16 ? TileCost{1, {3.85}, 0.9} : TileCost{1, {6.5}, 1.75};
}
inline double tile_us(const TileCost &c, long workgroups) {
    const long full = workgroups / (kUnits * c.most), rest = workgroups % (kUnits * c.most);
    return full * c.us[c.most - 1] + (rest > 0 ? c.us[(rest - 1) / kUnits] : 0.0);
}
}  // namespace scan_cost

struct ScanCut {
    int tiles, pieces, piece_tiles;                               // of a sequence; of a piece, the last one may have fewer
};
// The number of pieces with the least time: all of a sequence's tiles one after the other, or pieces of at least 4 tiles side by
// side after the kernel that forms their states (one piece fewer), a scan over the pieces and two more launches.
inline ScanCut scan_cut_of(int B, int N, int E, int G, int S, bool backward) {
    using namespace scan_cost;
    const int all = (N + kScanTile - 1) / kScanTile;
    const long whole = (long)B * scan_blocks(E, G);
    const TileCost c = backward ? bwd(S) : fwd(S);
    ScanCut cut{all, 1, all};
    double best = tile_us(c, whole) * all;
    for (int pieces = 2; pieces <= all / 4 && whole * pieces <= kUnits * c.most + whole; ++pieces) {
        const int tiles = (all + pieces - 1) / pieces;
        if ((all + tiles - 1) / tiles != pieces) continue;
        const double us = tiles * (tile_us(c, whole * pieces) + c.local * ((whole * (pieces - 1) + kUnits - 1) / kUnits)) + 10.0 + 0.25 * pieces;
        if (us < best) best = us, cut.pieces = pieces, cut.piece_tiles = tiles;
    }
    return cut;
}

}  // namespace la
