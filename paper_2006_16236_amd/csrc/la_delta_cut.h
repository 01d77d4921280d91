// How the gated delta rule cuts a sequence's chunks into pieces that run side by side (host code).
#pragma once

namespace la {

struct DeltaCut {
    int pieces, length;              // chunks a piece
};

// Workgroups that form transitions have no Q, M and outputs: two fit a compute unit, in registers, where heads are narrow (then
// 0.9 of a chunk's time for both, instead of 0.75 for one; training step of 2 x 4095 x 8 heads of 64 fp32: 223 -> 203 us).
constexpr bool two_lean(int bytes, int D) { return D == 32 || (D == 64 && bytes == 4); }

// A pass goes through the chunks of a head's 64 columns one after the other, one workgroup a compute unit.  Where there are
// few heads, pieces run side by side: a first launch takes the columns of V and, from the unit matrix, those of the
// transition of every piece but the first and the last (about 0.75 of a chunk's time, nothing is put out), a second one hands
// the states on, one product a piece, and the pass itself then starts every piece from its state.  In units of a chunk's time
// (2.2 to 3.7 us; a product of the join is 4.9 us for 128 x 128, 1.5 for 64 x 64); the cut with the least is taken, if it saves a
// tenth.  bytes: of an element of the tokens' tensors.
inline DeltaCut delta_cut_of(long heads, int D, int M, int chunks, int bytes) {
    const long blocks = (M + 63) / 64, across = (D + 63) / 64;
    const auto rounds = [](long workgroups, int places = 256) { return (double)((workgroups + places - 1) / places); };
    DeltaCut best{1, chunks};
    const double whole = rounds(heads * blocks) * chunks;
    double least = 0.9 * whole;
    for (int n = 2; n <= 64 && n <= chunks; ++n) {
        const int length = (chunks + n - 1) / n, pieces = (chunks + length - 1) / length;
        if (pieces != n) continue;
        const long firsts = heads * (blocks * (pieces - 1) + across * (pieces - 2));
        const double first = two_lean(bytes, D) && firsts > 256 ? 0.9 * length * rounds(firsts, 512) : 0.75 * length * rounds(firsts);
        const double join = 1.5 + (pieces > 2 ? 1.5 + (D == 128 ? 1.6 : 0.65) * (pieces - 2) * rounds(heads * blocks) : 0.0);
        const double cost = rounds(heads * blocks * pieces) * length + first + join;
        if (cost < least) least = cost, best = {pieces, length};
    }
    return best;
}

}  // namespace la
