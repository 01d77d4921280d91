// How the gated delta rule cuts a sequence's chunks into pieces that run side by side (host code).
#pragma once

namespace la {

struct DeltaCut {
    int pieces, length;              // chunks a piece
};

// A pass goes through the chunks of a head's 64 columns one after the other, one workgroup a compute unit.  Where there are
// few heads, pieces run side by side: a first launch takes the columns of V and, from the unit matrix, those of the
// transition of every piece but the first and the last (about 0.75 of a chunk's time, nothing is put out), a second one hands
// the states on, one product a piece, and the pass itself then starts every piece from its state.  In units of a chunk's time
// (2.2 to 3.7 us); the cut with the least is taken, if it saves a tenth.
inline DeltaCut delta_cut_of(long heads, int D, int M, int chunks) {
    const long blocks = (M + 63) / 64, across = (D + 63) / 64;
    const auto rounds = [](long workgroups) { return (double)((workgroups + 255) / 256); };
    DeltaCut best{1, chunks};
    const double whole = rounds(heads * blocks) * chunks;
    double least = 0.9 * whole;
    for (int n = 2; n <= 64 && n <= chunks; ++n) {
        const int length = (chunks + n - 1) / n, pieces = (chunks + length - 1) / length;
        if (pieces != n) continue;
        const double first = 0.75 * length * rounds(heads * (blocks * (pieces - 1) + across * (pieces - 2)));
        const double join = 1.5 + (pieces > 2 ? 1.5 + (pieces - 2) * rounds(heads * blocks) : 0.0);
        const double cost = rounds(heads * blocks * pieces) * length + first + join;
        if (cost < least) least = cost, best = {pieces, length};
    }
    return best;
}

}  // namespace la
