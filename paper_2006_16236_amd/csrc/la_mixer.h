// Arguments and launchers of the head norm with rotation (la_qk.hip) and of the gated delta rule (la_delta*.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>

#include "../../include/la.h"
#include "la_delta_cut.h"
#include "la_layer.h"

namespace la {

struct QkArgs {
    const void *q, *k, *dyq, *dyk;
    const float *wq, *wk, *freq;
    const int *pos, *lengths;
    void *yq, *yk;                   // backward: dq, dk
    float *part;                     // backward: [groups][2][D], or NULL
    long ldq, ldk;
    int B, N, H, Hk, D, R, norm, parts;
    bool adjacent;
    float eps;
};
int qk_groups(const QkArgs &a);
hipError_t launch_qk_fwd(QkArgs a, int dtype, hipStream_t s);
hipError_t launch_qk_bwd(QkArgs a, int dtype, hipStream_t s);

// A chunk of C tokens of one head ("unit"; unit = (b H + h) K + chunk, K chunks a sequence).
struct DeltaArgs {
    const void *q, *k, *v, *dO;
    const float *g, *beta, *h0, *dh1;
    const int *lengths;
    void *o, *dq, *dk, *dv;
    float *h1, *dh0, *dg, *dbeta;
    float *tri;                      // [unit][2][tri_floats(C)]: Z and the masked scores
    float *gate;                     // [unit][4][C]: exp of the decay since the chunk's start and until its end; its logarithm in two parts
    float *miss;                     // [unit][C][M]: what each token finds missing in the state, or NULL (not kept)
    float *state;                    // [unit][D][M]: the state before each chunk, or NULL
    float *write;                    // [unit][C][M]: backward, the gradient of what a token writes
    float *dstate;                   // [unit][D][M]: backward, the gradient of the state behind each chunk
    float *piece_state;              // [B H][pieces][D][M]: of a cut sequence, the state before each piece
    float *transition;               // [B H][pieces][D][D]: what a piece makes of the state before it
    float *piece_dstate;             // [B H][pieces][D][M]: backward, the gradient of the state behind each piece
    long ldq, ldk, ldv;
    int B, N, H, Hk, D, M, K, pieces, length;      // length: chunks a piece
    float scale;
};
// the lower 32 x 32 blocks of a C x C matrix, those of a block column behind each other
constexpr int tri_floats(int C) { return C == 64 ? 96 * 32 : 32 * 32; }
inline int delta_chunk(int dtype) { return dtype == 0 ? 32 : 64; }
// chunk-local matrices, then outputs, states and what is kept (o, h1, miss, state: each may be NULL)
hipError_t launch_delta_fwd(const DeltaArgs &a, int dtype, hipStream_t s);
hipError_t launch_delta_bwd(const DeltaArgs &a, int dtype, hipStream_t s);
// the states before (behind) the pieces of cut sequences from those that each piece leaves of none
void launch_join(const DeltaArgs &a, int dtype, bool back, hipStream_t s);
// one token of every sequence: h [B, H, D, M] in and out
hipError_t launch_delta_step(const DeltaArgs &a, float *h, int dtype, hipStream_t s);

}  // namespace la
