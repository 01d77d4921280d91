// Gated delta rule, backward (la_delta_bwd).
//
// With the notation of la_delta.hip (u: what a token finds missing, U = beta u), dO the gradient of the outputs and dS' that
// of the state behind a chunk, the gradient of what the tokens write, y, solves the transposed system:
//   dU = scale M^T dO + e^{G_C - G} K dS',   y = dU - Z^T beta dU,   dV = beta y,
//   dS = e^{G_C} dS' + scale Q^T e^G dO - K^T e^G dV.
// A first launch goes backwards through a sequence's chunks (16 columns of dS a wave, as the forward), and leaves y and the
// dS' of every chunk.  A second one takes all chunks side by side and contracts over the columns:
//   P = scale e^{G_t - G_s} dO U^T  (s <= t),   B = -e^{G_t - G_s} dV U^T  (s < t),
//   dQ = scale e^G dO S^T + P K,   dK = -e^G dV S^T + e^{G_C - G} U dS'^T + P^T Q + (B + B^T) K,
//   dbeta = y . u,   dg_t = sum of dG from t to the chunk's end,
//   dG_t = q . dQ - k . dK - 2 dV . (V - u),  and at the last token the whole <dS', S'> = e^{G_C} <dS', S> + sum k . e^{G_C - G} (U dS'^T).
// (G_t acts through every e^{G_t - ..} once with each sign: q . dQ and k . dK count them, and those of the system and of
// K S, in which a token stands on the reading side, twice with the wrong sign; these are dV . (V - u) together.)
#include <hip/hip_runtime.h>

#include "la_delta.h"

namespace la {
namespace {

// As the forward: 16 columns of dS' a wave; products that y does not wait for (Q^T e^G dO) run beside the cutting of values.
// The chain of products and the writes of dS', y and dV bound it: 8 x 2048 x 16 heads of 128 bf16, 470 MB written, 205 us.
template <typename T, int D, PassKind kKind> __global__ __launch_bounds__(512) void delta_states_bwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks, kSteps = D / 32;
    constexpr bool kOutputs = kKind == kWhole;
    __shared__ Chunked<T, D> buffers[2];
    Task task;
    if (!task_of<kKind, true>(a, C, D, task)) return;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), c = lane % 16, g = lane / 16, m = task.m0 + wave * 16 + c;
    const int h = task.h, len = task.len, count = task.count, ldo = a.H * a.M;
    const size_t seq = (size_t)task.b * a.N, state = (size_t)task.bh * D * a.M, piece = (size_t)task.bh * a.pieces + task.piece;
    if (wave >= 4) {
        fetch_chunks<T, D, false, true>(buffers, a, task, (const T *)a.dO, ldo, tid - 256);
        return;
    }
    if (wave * 16 >= task.cols) {
        if (count > 0) __syncthreads();
        for (int i = 0; i < count; ++i) __syncthreads();
        return;
    }
    f32x4 S[D / 16];                                         // dS'
    const float *from = task.end ? (a.dh1 == nullptr ? nullptr : a.dh1 + state) : kOutputs ? a.piece_dstate + piece * D * a.M : nullptr;
    load_state<D>(from, m, a.M, g, S);
    loads_done();
    Parts<3> sp[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sp[s] = cut(S[2 * s], S[2 * s + 1]);
    if (kOutputs && task.end)
        for (int n = len + g; n < a.N; n += 4) store_elem<false>((T *)a.dv + (seq + n) * ldo + (size_t)h * a.M + m, 0.0f);      // tokens behind the sequence
    if (count > 0) __syncthreads();
    for (int i = 0; i < count; ++i) {
        const int chunk = task.first + count - 1 - i, left = len - chunk * C;
        const long unit = (long)task.bh * a.K + chunk;
        const Chunked<T, D> &in = buffers[i & 1];
        const auto gate4 = [&](int which, int t) { return *reinterpret_cast<const f32x4 *>(in.gates + which * C + paired(t, 4 * g)); };
        f32x4 y[kTiles], w[kTiles];
        Parts<P> f[2][kTiles], o[kBlocks];
        Raw4<P> out[kTiles];
        const auto rows = [&](int s) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) f[s % 2][t] = row_operand<D, P>(in.k, C * D, paired(t, c), 4 * s + g);
        };
        // a block column's tiles of a transposed chunk-local matrix
        const auto upper = [&](const uint16_t *mat, Parts<3> (&tri)[kTiles][kBlocks]) {
#pragma unroll
            for (int s = 0; s < kBlocks; ++s)
#pragma unroll
                for (int t = 0; t < 2 * (s + 1); ++t) tri[t][s] = column_operand<32, true, 3>(mat, Ch::kTri, tri_row<C>(32 * s, t / 2), t % 2, lane);
        };
        Parts<3> tri[kTiles][kBlocks];
        rows(0);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = w[t] = f32x4{0, 0, 0, 0};
        if constexpr (kOutputs) store_state<D>(a.dstate + (size_t)unit * D * a.M, m - c, a.M, lane, S);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s + 1 < kSteps) rows(s + 1);
            else {
#pragma unroll
                for (int x = 0; x < kBlocks; ++x) o[x] = column_operand<kCols, false, P>(in.v, C * kCols, 32 * x, wave, lane);
                upper(in.m, tri);
            }
            in_this_order<D>();
            products(f[s % 2], sp[s], y);
        }
        in_this_order<D>();
#pragma unroll
        for (int t = 0; t < kTiles; ++t) out[t] = column_values<kCols, P>(in.v, C * kCols, paired(t, 4 * g), wave, lane);
        upper_products(tri, o, w);
        in_this_order<D>();
        // dU, and beside it the state's share of the outputs
        constexpr int kGroup = 4 < D / 16 ? 4 : D / 16, kGroups = D / 16 / kGroup;
        Parts<P> kt[2][kGroup];
        const auto columns = [&](const uint16_t *mat, int n) {
#pragma unroll
            for (int t = 0; t < kGroup; ++t) kt[n % 2][t] = column_operand<D, true, P>(mat, C * D, 32 * (n % kBlocks), n / kBlocks * kGroup + t, lane);
        };
        const float whole = in.gates[C - 1];
        Parts<3> x[kBlocks], z[kBlocks];
#pragma unroll
        for (int s = 0; s < kBlocks; ++s)
            x[s] = cut(a.scale * gate4(0, 2 * s) * out[2 * s].sum(), a.scale * gate4(0, 2 * s + 1) * out[2 * s + 1].sum());
#pragma unroll
        for (int t = 0; t < D / 16; ++t) S[t] *= whole;
        columns(in.q, 0);
        in_this_order<D>();
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = a.scale * w[t] + gate4(1, t) * y[t], w[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) z[s] = cut(gate4(2, 2 * s) * y[2 * s], gate4(2, 2 * s + 1) * y[2 * s + 1]);
        const auto update = [&](int n, const Parts<3> &by) {
            f32x4 part[kGroup];
#pragma unroll
            for (int t = 0; t < kGroup; ++t) part[t] = S[n / kBlocks * kGroup + t];
            products(kt[n % 2], by, part);
#pragma unroll
            for (int t = 0; t < kGroup; ++t) S[n / kBlocks * kGroup + t] = part[t];
        };
#pragma unroll
        for (int n = 0; n < kGroups * kBlocks; ++n) {
            if (n + 1 < kGroups * kBlocks) columns(in.q, n + 1);
            update(n, x[n % kBlocks]);
            if (n == 0) side_by_side<D, kGroup * (P == 1 ? 3 : 6)>();
            in_this_order<D>();
        }
        upper(in.z, tri);
        upper_products(tri, z, w);
        columns(in.k, 0);
        in_this_order<D>();
        const Range wr = range_of(a.write + (size_t)unit * C * a.M, C, a.M, a.M);
        const Range vr = range_of((T *)a.dv + (seq + (size_t)chunk * C) * ldo + (size_t)h * a.M, left < C ? left : C, ldo, a.M);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] -= w[t], w[t] = gate4(2, t) * y[t];       // w: dV
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x[s] = cut(-gate4(0, 2 * s) * w[2 * s], -gate4(0, 2 * s + 1) * w[2 * s + 1]);
        in_this_order<D>();
#pragma unroll
        for (int n = 0; n < kGroups * kBlocks; ++n) {
            if (n + 1 < kGroups * kBlocks) columns(in.k, n + 1);
            update(n, x[n % kBlocks]);
            if (kOutputs && n == 0) {
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    store_tile<float>(wr, paired(t, 4 * g), m - c, a.M, y[t], lane);
                    store_tile<T>(vr, paired(t, 4 * g), m - c, ldo, w[t], lane);
                }
            }
            if (n % kBlocks == 0 && n > 0) {                 // the group before is complete
#pragma unroll
                for (int s = 0; s < kGroup / 2; ++s) {
                    const int j = (n / kBlocks - 1) * kGroup / 2 + s;
                    sp[j] = cut(S[2 * j], S[2 * j + 1]);
                }
            }
            if (n % kBlocks == 0) side_by_side<D, kGroup * (P == 1 ? 3 : 6)>();
            in_this_order<D>();
        }
#pragma unroll
        for (int j = (kGroups - 1) * kGroup / 2; j < kSteps; ++j) sp[j] = cut(S[2 * j], S[2 * j + 1]);
        __syncthreads();
    }
    if constexpr (!kOutputs) store_state<D>(a.piece_dstate + (piece - 1) * D * a.M, m - c, a.M, lane, S);
    else if (task.start && a.dh0 != nullptr) store_state<D>(a.dh0 + state, m - c, a.M, lane, S);
}

// A workgroup takes one chunk and the heads that share its queries and keys, one after the other; a wave has kSlabs times 16
// columns of dQ and dK; the columns of the states come 32 at a time ("turn").  What a turn reads from memory is on its way
// during the turn before, and two workgroups share a compute unit: with all columns of eight waves at once, one workgroup, half
// of the time went to waiting for loads (8 x 2048 x 16 heads of 128 bf16: 462 us, now 370: 1.18 GB, 3.2 TB/s).
// kShared: sums over more than one head wait in LDS.
template <typename T, int D, bool kShared> __global__ __launch_bounds__(D == 32 ? 128 : 256, kShared && D != 64 ? 1 : 2) void delta_chunks_bwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks, kWaves = D == 32 ? 2 : 4, kThreads = 64 * kWaves;
    constexpr int kSlabs = D / 16 / kWaves, kTurn = 32, kPieces = kTurn / 8;
    constexpr int kLow = kTiles * (kTiles + 1) / 2, kLowEach = (kLow + kWaves - 1) / kWaves;
    constexpr int kStage = (6 + P) * C * kTurn, kSquare = 3 * C * C, kWork = kStage > kSquare ? kStage : kSquare;
    constexpr int kEach = (C * kPieces + kThreads - 1) / kThreads, kGateEach = (4 * C + kThreads - 1) / kThreads;
    __shared__ alignas(16) uint16_t kS[P * C * D], qS[P * C * D], work[kWork];
    __shared__ alignas(16) float gates[4 * C], bt[C], miss[C], db[C], red[kWaves][C], ends[kWaves];
    __shared__ f32x4 sums[kShared ? 2 : 1][kShared ? kSlabs * kTiles : 1][kShared ? kThreads : 1];      // dQ, dK so far
    uint16_t *uS = work, *wS = work + 3 * C * kTurn, *oS = work + 6 * C * kTurn, *square = work;          // U, dV, dO; P, then B
    int tid = threadIdx.x, lane = tid % kWave, c = lane % 16, g = lane / 16;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int chunk = (int)(blockIdx.x % a.K), bk = (int)(blockIdx.x / a.K), b = bk / a.Hk, hk = bk % a.Hk, per = a.H / a.Hk;
    const int len = length_of(a, b), t0 = chunk * C, left = len - t0, rows = left < C ? left : C, ldo = a.H * a.M;
    const size_t row0 = (size_t)b * a.N + t0;
    const int inside = a.N - t0 < C ? a.N - t0 : C, ldd = a.Hk * D;
    const Range dqr = range_of((T *)a.dq + row0 * ldd + (size_t)hk * D, inside, ldd, D), dkr = range_of((T *)a.dk + row0 * ldd + (size_t)hk * D, inside, ldd, D);
    if (left <= 0) {                                         // behind the sequence
        for (int i = tid; i < C * per; i += kThreads) {
            const int t = i / per;
            const size_t at = (row0 + t) * a.H + hk * per + i % per;
            if (t0 + t >= a.N) break;
            if (a.dg != nullptr) a.dg[at] = 0.0f;
            a.dbeta[at] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < kSlabs * kTiles; ++i) {
            store_tile<T>(dqr, 16 * (i % kTiles) + 4 * g, 16 * (wave * kSlabs + i / kTiles), ldd, f32x4{0, 0, 0, 0}, lane);
            store_tile<T>(dkr, 16 * (i % kTiles) + 4 * g, 16 * (wave * kSlabs + i / kTiles), ldd, f32x4{0, 0, 0, 0}, lane);
        }
        return;
    }
    const int turns = (a.M + kTurn - 1) / kTurn, all = per * turns;
    // what one turn reads: u, y, V, dO of its columns, S and dS' of this lane's rows
    Eight<float> us[kEach], ys[kEach], s0[kSlabs], s1[kSlabs];
    Eight<T> vs[kEach], os[kEach];
    float gate_in[kGateEach], beta_in;
    const auto load = [&](int turn) {
        const int n = turn < all ? turn : 0, h = hk * per + n / turns, m0 = n % turns * kTurn;
        const int cols = turn >= all ? 0 : a.M - m0 < kTurn ? a.M - m0 : kTurn;          // nothing behind the last turn
        const long unit = (long)(b * a.H + h) * a.K + chunk;
        const Range ur = range_of(a.miss + (size_t)unit * C * a.M + m0, C, a.M, cols), yr = range_of(a.write + (size_t)unit * C * a.M + m0, C, a.M, cols);
        const Range vr = range_of((const T *)a.v + row0 * a.ldv + (size_t)h * a.M + m0, rows, a.ldv, cols);
        const Range zr = range_of((const T *)a.dO + row0 * ldo + (size_t)h * a.M + m0, rows, ldo, cols);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = tid + kThreads * j, t = i / kPieces, piece = i % kPieces;
            const bool in = 8 * piece < cols && (C * kPieces % kThreads == 0 || i < C * kPieces);
            us[j] = load_eight<float>(ur, in ? (t * a.M + 8 * piece) * 4 : 0x7fffff00);
            ys[j] = load_eight<float>(yr, in ? (t * a.M + 8 * piece) * 4 : 0x7fffff00);
            vs[j] = load_eight<T>(vr, in ? (t * (int)a.ldv + 8 * piece) * (int)sizeof(T) : 0x7fffff00);
            os[j] = load_eight<T>(zr, in ? (t * ldo + 8 * piece) * (int)sizeof(T) : 0x7fffff00);
        }
        const Range br = range_of(a.beta + row0 * a.H + h, rows, a.H, 1);
#pragma unroll
        for (int j = 0; j < kGateEach; ++j) gate_in[j] = a.gate[unit * 4 * C + (tid + kThreads * j) % (4 * C)];
        beta_in = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(br, tid * a.H * 4, 0, 0));
    };
    const auto load_states = [&](int n) {
        const int h = hk * per + n / turns, m0 = n % turns * kTurn, cols = a.M - m0 < kTurn ? a.M - m0 : kTurn;
        const size_t at = (size_t)((long)(b * a.H + h) * a.K + chunk) * D * a.M + m0;
        const Range s0r = range_of(a.state + at, D, a.M, cols), s1r = range_of(a.dstate + at, D, a.M, cols);
#pragma unroll
        for (int x = 0; x < kSlabs; ++x) {
            const int in = 8 * g < cols ? ((16 * (wave * kSlabs + x) + c) * a.M + 8 * g) * 4 : 0x7fffff00;
            s0[x] = load_eight<float>(s0r, in), s1[x] = load_eight<float>(s1r, in);
        }
    };
    {
        constexpr int kTok = C * D / 8, kTokEach = (kTok + kThreads - 1) / kThreads;
        const Range kr = range_of((const T *)a.k + row0 * a.ldk + (size_t)hk * D, rows, a.ldk, D);
        const Range qr = range_of((const T *)a.q + row0 * a.ldq + (size_t)hk * D, rows, a.ldq, D);
        Eight<T> kq[kTokEach][2];
#pragma unroll
        for (int j = 0; j < kTokEach; ++j) {
            const int i = tid + kThreads * j, t = i / (D / 8), piece = i % (D / 8);
            kq[j][0] = load_eight<T>(kr, (t * (int)a.ldk + 8 * piece) * (int)sizeof(T));
            kq[j][1] = load_eight<T>(qr, (t * (int)a.ldq + 8 * piece) * (int)sizeof(T));
        }
        load(0);
#pragma unroll
        for (int j = 0; j < kTokEach; ++j) {
            const int i = tid + kThreads * j, t = i / (D / 8), piece = i % (D / 8);
            park_eight<T>(kS + mat_at<D, true>(t, piece), C * D, kq[j][0]);
            park_eight<T>(qS + mat_at<D, true>(t, piece), C * D, kq[j][1]);
        }
    }
    f32x4 q1[kSlabs][kTiles], k1[kSlabs][kTiles], k2[kSlabs][kTiles], p[kLowEach], bb[kLowEach];
    float both = 0.0f;                                       // <S, dS'>
    // the wave's tiles of a lower triangle: columns 16 st .. of s, rows 16 ct .. of t; where it has fewer, the last one again, not stored
    int st[kLowEach], ct[kLowEach];
#pragma unroll
    for (int i = 0; i < kLowEach; ++i) {
        const int at = wave + i * kWaves < kLow ? wave + i * kWaves : kLow - 1;
        ct[i] = at < 1 ? 0 : at < 3 ? 1 : at < 6 ? 2 : 3, st[i] = at - ct[i] * (ct[i] + 1) / 2;
    }
    const auto own = [&](int i) { return wave + i * kWaves < kLow; };
    for (int n = 0; n < all; ++n) {
        const int h = hk * per + n / turns;
        load_states(n);
        tid = here(tid), lane = tid % kWave, c = lane % 16, g = lane / 16;
        __syncthreads();                                     // the turn before has been read
        if (n % turns == 0) {
#pragma unroll
            for (int j = 0; j < kGateEach; ++j)
                if (tid + kThreads * j < 4 * C) gates[tid + kThreads * j] = gate_in[j];
            if (tid < C) bt[tid] = beta_in, miss[tid] = db[tid] = 0.0f;
            __syncthreads();
            both = 0.0f;
#pragma unroll
            for (int x = 0; x < kSlabs; ++x)
#pragma unroll
                for (int t = 0; t < kTiles; ++t) q1[x][t] = k1[x][t] = k2[x][t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kLowEach; ++i) p[i] = bb[i] = f32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int i = tid + kThreads * j, t = i / kPieces, piece = i % kPieces;
            if (C * kPieces % kThreads != 0 && i >= C * kPieces) break;
            float u[8], w[8], dots = 0.0f, dbs = 0.0f;
            const float beta = bt[t];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[e] = beta * us[j].get(e), w[e] = beta * ys[j].get(e);
                dots = fmaf(w[e], vs[j].get(e) - us[j].get(e), dots);
                dbs = fmaf(ys[j].get(e), us[j].get(e), dbs);
            }
            const int at = mat_at<kTurn, true>(t, piece);
            park_eight(uS + at, C * kTurn, u);
            park_eight(wS + at, C * kTurn, w);
            park_eight<T>(oS + at, C * kTurn, os[j]);
            dots += dpp_move<0xB1>(dots), dbs += dpp_move<0xB1>(dbs);           // over the four lanes of a token
            dots += dpp_move<0x4E>(dots), dbs += dpp_move<0x4E>(dbs);
            if (piece == 0) miss[t] += dots, db[t] += dbs;
        }
        load(n + 1);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLowEach; ++i) {                 // P^T and B^T: rows s, columns t >= s
            const Parts<3> u = row_operand<kTurn, 3, true>(uS, C * kTurn, 16 * st[i] + c, g);
            p[i] = product(u, row_operand<kTurn, P, true>(oS, C * kTurn, 16 * ct[i] + c, g), p[i]);
            bb[i] = product(u, row_operand<kTurn, 3, true>(wS, C * kTurn, 16 * ct[i] + c, g), bb[i]);
        }
#pragma unroll
        for (int x = 0; x < kSlabs; ++x) {                   // one after the other: their operands together are too many registers
#pragma unroll
            for (int e = 0; e < 8; ++e) both = fmaf(s0[x].get(e), s1[x].get(e), both);
            const Parts<3> x0 = cut(f32x4{s0[x].get(0), s0[x].get(1), s0[x].get(2), s0[x].get(3)}, f32x4{s0[x].get(4), s0[x].get(5), s0[x].get(6), s0[x].get(7)});
            const Parts<3> x1 = cut(f32x4{s1[x].get(0), s1[x].get(1), s1[x].get(2), s1[x].get(3)}, f32x4{s1[x].get(4), s1[x].get(5), s1[x].get(6), s1[x].get(7)});
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                q1[x][t] = product(row_operand<kTurn, P, true>(oS, C * kTurn, 16 * t + c, g), x0, q1[x][t]);
                k1[x][t] = product(row_operand<kTurn, 3, true>(wS, C * kTurn, 16 * t + c, g), x0, k1[x][t]);
                k2[x][t] = product(row_operand<kTurn, 3, true>(uS, C * kTurn, 16 * t + c, g), x1, k2[x][t]);
                if (kSlabs > 1 && t % 2 == 1) in_this_order();
            }
        }
        if (n % turns != turns - 1) continue;
        tid = here(tid), lane = tid % kWave, c = lane % 16, g = lane / 16;
        __syncthreads();                                     // U, dV, dO make way for P
        // rows t, columns s of a lower triangle in LDS
        const auto park_low = [&](int i, const float (&v)[4]) {
            const int t = 16 * ct[i] + c, s = 16 * st[i] + 4 * g;
            const Split3 w = split3(v);
            const u32x2_t parts[3] = {w.h, w.m, w.l};
#pragma unroll
            for (int k = 0; k < 3; ++k) *reinterpret_cast<u32x2_t *>(square + k * C * C + mat_at<C, true>(t, s / 8) + s % 8) = parts[k];
        };
#pragma unroll
        for (int i = 0; i < kLowEach; ++i) {
            const int t = 16 * ct[i] + c, s = 16 * st[i] + 4 * g;
            const f32x4 hi = gates[2 * C + t] - *reinterpret_cast<const f32x4 *>(gates + 2 * C + s), lo = gates[3 * C + t] - *reinterpret_cast<const f32x4 *>(gates + 3 * C + s);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float decay = s + r <= t ? decay_of(hi[r], lo[r]) : 0.0f;
                p[i][r] = s + r <= t ? a.scale * p[i][r] * decay : 0.0f;
                bb[i][r] = s + r < t ? -bb[i][r] * decay : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < kLowEach; ++i) {
            if (!own(i)) break;
            park_low(i, {p[i][0], p[i][1], p[i][2], p[i][3]});
            // the tile right above the diagonal, which products over 32 tokens read
            if (st[i] == ct[i] && ct[i] % 2 == 0)
#pragma unroll
                for (int k = 0; k < 3; ++k) *reinterpret_cast<u32x2_t *>(square + k * C * C + mat_at<C, true>(16 * ct[i] + c, 2 * st[i] + 2 + g / 2) + 4 * (g & 1)) = u32x2_t{0, 0};
        }
        __syncthreads();
        float into = 0.0f;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const f32x4 eg = *reinterpret_cast<const f32x4 *>(gates + 16 * t + 4 * g), eh = *reinterpret_cast<const f32x4 *>(gates + C + 16 * t + 4 * g);
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) {
                const f32x4 kv = column_values<D, P, true>(kS, C * D, 16 * t + 4 * g, wave * kSlabs + x, lane).sum();
                k2[x][t] = eh * k2[x][t];
#pragma unroll
                for (int r = 0; r < 4; ++r) into = fmaf(kv[r], k2[x][t][r], into);
                q1[x][t] = a.scale * eg * q1[x][t];
                k1[x][t] = k2[x][t] - eg * k1[x][t];
            }
            if (kSlabs > 1) in_this_order();
        }
        // products with a lower triangle in LDS, from the left: with its rows, and with its columns
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) {
            Parts<P> kx[kSlabs], qx[kSlabs];
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) {
                kx[x] = column_operand<D, false, P, true>(kS, C * D, 32 * s, wave * kSlabs + x, lane);
                qx[x] = column_operand<D, false, P, true>(qS, C * D, 32 * s, wave * kSlabs + x, lane);
            }
#pragma unroll
            for (int t = 2 * s; t < kTiles; ++t) {
                const Parts<3> f = row_operand<C, 3, true>(square, C * C, 16 * t + c, 4 * s + g);
#pragma unroll
                for (int x = 0; x < kSlabs; ++x) q1[x][t] = product(f, kx[x], q1[x][t]);
                if (kSlabs > 1 && t % 2 == 1) in_this_order();
            }
#pragma unroll
            for (int t = 0; t < 2 * (s + 1); ++t) {
                const Parts<3> f = column_operand<C, false, 3, true>(square, C * C, 32 * s, t, lane);
#pragma unroll
                for (int x = 0; x < kSlabs; ++x) k1[x][t] = product(f, qx[x], k1[x][t]);
                if (kSlabs > 1 && t % 2 == 1) in_this_order();
            }
        }
        __syncthreads();                                     // P makes way for B
#pragma unroll
        for (int i = 0; i < kLowEach; ++i) {
            if (!own(i)) break;
            park_low(i, {bb[i][0], bb[i][1], bb[i][2], bb[i][3]});
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) {
            Parts<P> kx[kSlabs];
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) kx[x] = column_operand<D, false, P, true>(kS, C * D, 32 * s, wave * kSlabs + x, lane);
#pragma unroll
            for (int t = 2 * s; t < kTiles; ++t) {
                const Parts<3> f = row_operand<C, 3, true>(square, C * C, 16 * t + c, 4 * s + g);
#pragma unroll
                for (int x = 0; x < kSlabs; ++x) k1[x][t] = product(f, kx[x], k1[x][t]);
                if (kSlabs > 1 && t % 2 == 1) in_this_order();
            }
#pragma unroll
            for (int t = 0; t < 2 * (s + 1); ++t) {
                const Parts<3> f = column_operand<C, false, 3, true>(square, C * C, 32 * s, t, lane);
#pragma unroll
                for (int x = 0; x < kSlabs; ++x) k1[x][t] = product(f, kx[x], k1[x][t]);
                if (kSlabs > 1 && t % 2 == 1) in_this_order();
            }
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f32x4 dot = {0, 0, 0, 0};
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) {
                const int slab = wave * kSlabs + x;
                f32x4 qd = q1[x][t], kd = k1[x][t];
                dot += column_values<D, P, true>(qS, C * D, 16 * t + 4 * g, slab, lane).sum() * qd - column_values<D, P, true>(kS, C * D, 16 * t + 4 * g, slab, lane).sum() * kd;
                if constexpr (kShared) {
                    if (h > hk * per) qd += sums[0][x * kTiles + t][tid], kd += sums[1][x * kTiles + t][tid];
                    sums[0][x * kTiles + t][tid] = qd, sums[1][x * kTiles + t][tid] = kd;
                }
                if (n == all - 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * t + 4 * g + r >= left) qd[r] = kd[r] = 0.0f;
                    store_tile<T>(dqr, 16 * t + 4 * g, 16 * slab, ldd, qd, lane);
                    store_tile<T>(dkr, 16 * t + 4 * g, 16 * slab, ldd, kd, lane);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float v = row_sum16(dot[r]);
                if (c == 0) red[wave][16 * t + 4 * g + r] = v;
            }
            if (kSlabs > 1) in_this_order();
        }
        into = wave_sum(fmaf(gates[C - 1], both, into));
        if (lane == 0) ends[wave] = into;
        __syncthreads();
        if (wave == 0) {
            double sum = 0.0;
            if (lane < C) {
                sum = -2.0 * (double)miss[lane];
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    sum += (double)red[w][lane];
                    if (lane == C - 1) sum += (double)ends[w];
                }
            }
#pragma unroll
            for (int k = 1; k < C; k *= 2) {
                const double from = __shfl_down(sum, k);
                if (lane + k < C) sum += from;
            }
            if (lane < C && t0 + lane < a.N) {
                const size_t at = (row0 + lane) * a.H + h;
                if (a.dg != nullptr) a.dg[at] = lane < left ? (float)sum : 0.0f;
                a.dbeta[at] = lane < left ? db[lane] : 0.0f;
            }
        }
    }
}
}  // namespace

hipError_t launch_delta_bwd(const DeltaArgs &a, int dtype, hipStream_t s) {
    if (a.pieces > 1) {
#define LA_PIECES(T, D) delta_states_bwd_kernel<T, D, kStates><<<task_grid(a, kStates), 512, 0, s>>>(a)
        LA_BY_WIDTH(LA_PIECES)
        if (a.pieces > 2) launch_join(a, dtype, true, s);
    }
#define LA_STATES(T, D) delta_states_bwd_kernel<T, D, kWhole><<<task_grid(a, kWhole), 512, 0, s>>>(a)
    LA_BY_WIDTH(LA_STATES)
    const unsigned units = (unsigned)((long)a.B * a.Hk * a.K);
#define LA_CHUNKS(T, D) a.H > a.Hk ? delta_chunks_bwd_kernel<T, D, true><<<units, D == 32 ? 128 : 256, 0, s>>>(a) : delta_chunks_bwd_kernel<T, D, false><<<units, D == 32 ? 128 : 256, 0, s>>>(a)
    LA_BY_WIDTH(LA_CHUNKS)
    return hipGetLastError();
}

}  // namespace la
