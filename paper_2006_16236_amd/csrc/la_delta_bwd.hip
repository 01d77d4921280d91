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
template <typename T, int D> __global__ __launch_bounds__(512) void delta_states_bwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks, kSteps = D / 32;
    __shared__ Chunked<T, D> buffers[2];
    int bh, m0;
    if (!head_and_columns(a, bh, m0)) return;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, c = lane % 16, g = lane / 16, m = m0 + wave * 16 + c;
    const int b = bh / a.H, h = bh % a.H, len = length_of(a, b), chunks = (len + C - 1) / C;
    const int cols = a.M - m0 < kCols ? a.M - m0 : kCols, ldo = a.H * a.M;
    const size_t seq = (size_t)b * a.N, state = (size_t)bh * D * a.M;
    if (wave >= 4) {
        fetch_chunks<T, D>(buffers, a, bh, len, chunks - 1, -1, chunks, (const T *)a.dO + (size_t)h * a.M + m0, ldo, cols, tid - 256);
        return;
    }
    if (wave * 16 >= cols) {
        if (chunks > 0) __syncthreads();
        for (int chunk = 0; chunk < chunks; ++chunk) __syncthreads();
        return;
    }
    f32x4 S[D / 16];                                         // dS'
    load_state<D>(a.dh1 == nullptr ? nullptr : a.dh1 + state, m, a.M, g, S);
    loads_done();
    Parts<3> sp[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sp[s] = cut(S[2 * s], S[2 * s + 1]);
    for (int n = len + g; n < a.N; n += 4) store_elem<false>((T *)a.dv + (seq + n) * ldo + (size_t)h * a.M + m, 0.0f);      // tokens behind the sequence
    if (chunks > 0) __syncthreads();
    for (int i = 0; i < chunks; ++i) {
        const int chunk = chunks - 1 - i, left = len - chunk * C;
        const long unit = (long)bh * a.K + chunk;
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
        store_state<D>(a.dstate + (size_t)unit * D * a.M, m - c, a.M, lane, S);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s + 1 < kSteps) rows(s + 1);
            else {
#pragma unroll
                for (int x = 0; x < kBlocks; ++x) o[x] = column_operand<kCols, false, P>(in.v, C * kCols, 32 * x, wave, lane);
                upper(in.m, tri);
            }
            in_this_order();
            products(f[s % 2], sp[s], y);
        }
        in_this_order();
#pragma unroll
        for (int t = 0; t < kTiles; ++t) out[t] = column_values<kCols, P>(in.v, C * kCols, paired(t, 4 * g), wave, lane);
        upper_products<2>(tri, o, w);
        in_this_order();
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
        in_this_order();
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
            if (n == 0) side_by_side<kGroup * (P == 1 ? 3 : 6)>();
            in_this_order();
        }
        upper(in.z, tri);
        upper_products<2>(tri, z, w);
        columns(in.k, 0);
        in_this_order();
        const Range wr = range_of(a.write + (size_t)unit * C * a.M, C, a.M, a.M);
        const Range vr = range_of((T *)a.dv + (seq + (size_t)chunk * C) * ldo + (size_t)h * a.M, left < C ? left : C, ldo, a.M);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] -= w[t], w[t] = gate4(2, t) * y[t];       // w: dV
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x[s] = cut(-gate4(0, 2 * s) * w[2 * s], -gate4(0, 2 * s + 1) * w[2 * s + 1]);
        in_this_order();
#pragma unroll
        for (int n = 0; n < kGroups * kBlocks; ++n) {
            if (n + 1 < kGroups * kBlocks) columns(in.k, n + 1);
            update(n, x[n % kBlocks]);
            if (n == 0) {
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
            if (n % kBlocks == 0) side_by_side<kGroup * (P == 1 ? 3 : 6)>();
            in_this_order();
        }
#pragma unroll
        for (int j = (kGroups - 1) * kGroup / 2; j < kSteps; ++j) sp[j] = cut(S[2 * j], S[2 * j + 1]);
        __syncthreads();
    }
    if (a.dh0 != nullptr) store_state<D>(a.dh0 + state, m - c, a.M, lane, S);
}

// A workgroup takes one chunk and the heads that share its queries and keys, one after the other, D / 16 waves with 16
// columns of dQ and dK each; the columns of the states 64 at a time.
template <typename T, int D> __global__ __launch_bounds__(4 * D) void delta_chunks_bwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks, kWaves = D / 16, kThreads = 4 * D;
    constexpr int kLow = kTiles * (kTiles + 1) / 2, kLowEach = (kLow + kWaves - 1) / kWaves;
    constexpr int kStage = (6 + P) * C * kCols, kSquares = 6 * C * C, kWork = kStage > kSquares ? kStage : kSquares;
    __shared__ alignas(16) uint16_t kS[P * C * D], qS[P * C * D], work[kWork];
    __shared__ alignas(16) float gates[4 * C], bt[C], miss[C], db[C], red[kWaves][C], ends[kWaves];
    uint16_t *uS = work, *wS = work + 3 * C * kCols, *oS = work + 6 * C * kCols;          // U, dV, dO
    uint16_t *pS = work, *bS = work + 3 * C * C;                                            // P, B + B^T
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, c = lane % 16, g = lane / 16, d = 16 * wave + c;
    const int chunk = (int)(blockIdx.x % a.K), bk = (int)(blockIdx.x / a.K), b = bk / a.Hk, hk = bk % a.Hk, per = a.H / a.Hk;
    const int len = length_of(a, b), t0 = chunk * C, left = len - t0;
    const size_t row0 = (size_t)b * a.N + t0, ldo = (size_t)a.H * a.M;
    f32x4 dq[kTiles], dk[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) dq[t] = dk[t] = f32x4{0, 0, 0, 0};
    if (left > 0) {
        for (int i = tid; i < C * D / 8; i += kThreads) {
            const int t = i / (D / 8), piece = i % (D / 8);
            park_eight<T>(kS + mat_at<D, true>(t, piece), C * D, load_eight<T>((const T *)a.k + (row0 + t) * a.ldk + (size_t)hk * D + 8 * piece, t < left));
            park_eight<T>(qS + mat_at<D, true>(t, piece), C * D, load_eight<T>((const T *)a.q + (row0 + t) * a.ldq + (size_t)hk * D + 8 * piece, t < left));
        }
        for (int h = hk * per; h < (hk + 1) * per; ++h) {
            const long unit = (long)(b * a.H + h) * a.K + chunk;
            __syncthreads();                                 // the head before is done with everything below
            for (int i = tid; i < 4 * C; i += kThreads) gates[i] = a.gate[unit * 4 * C + i];
            for (int i = tid; i < C; i += kThreads) bt[i] = i < left ? a.beta[(row0 + i) * a.H + h] : 0.0f, miss[i] = db[i] = 0.0f;
            f32x4 q1[kTiles], k1[kTiles], k2[kTiles], p[kLowEach], bb[kLowEach];
            float both = 0.0f;                               // <S, dS'>
#pragma unroll
            for (int t = 0; t < kTiles; ++t) q1[t] = k1[t] = k2[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kLowEach; ++i) p[i] = bb[i] = f32x4{0, 0, 0, 0};
            for (int m0 = 0; m0 < a.M; m0 += kCols) {
                __syncthreads();
                for (int i = tid; i < C * 8; i += kThreads) {
                    const int t = i / 8, piece = i % 8, m = m0 + 8 * piece;
                    const bool have = m < a.M, live = have && t < left;
                    const Eight<float> us = load_eight<float>(a.miss + ((size_t)unit * C + t) * a.M + m, have);
                    const Eight<float> ys = load_eight<float>(a.write + ((size_t)unit * C + t) * a.M + m, have);
                    const Eight<T> vs = load_eight<T>((const T *)a.v + (row0 + t) * a.ldv + (size_t)h * a.M + m, live);
                    const Eight<T> os = load_eight<T>((const T *)a.dO + (row0 + t) * ldo + (size_t)h * a.M + m, live);
                    float u[8], w[8], dots = 0.0f, dbs = 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        u[e] = bt[t] * us.get(e), w[e] = bt[t] * ys.get(e);
                        dots = fmaf(w[e], vs.get(e) - us.get(e), dots);
                        dbs = fmaf(ys.get(e), us.get(e), dbs);
                    }
                    const int at = mat_at<kCols, true>(t, piece);
                    park_eight(uS + at, C * kCols, u);
                    park_eight(wS + at, C * kCols, w);
                    park_eight<T>(oS + at, C * kCols, os);
                    dots += dpp_move<0xB1>(dots), dbs += dpp_move<0xB1>(dbs);       // over the eight lanes of a token
                    dots += dpp_move<0x4E>(dots), dbs += dpp_move<0x4E>(dbs);
                    dots += dpp_move<0x141>(dots), dbs += dpp_move<0x141>(dbs);
                    if (piece == 0) miss[t] += dots, db[t] += dbs;
                }
                __syncthreads();
                // tiles of P^T and B^T: rows s, columns t >= s
#pragma unroll
                for (int i = 0; i < kLowEach; ++i) {
                    int n = wave + i * kWaves, ct = 0;
                    if (n >= kLow) break;
                    while (n > ct) n -= ++ct;                // n-th tile s of column tile t = ct
#pragma unroll
                    for (int s = 0; s < kCols / 32; ++s) {
                        const Parts<3> u = row_operand<kCols, 3, true>(uS, C * kCols, 16 * n + c, 4 * s + g);
                        p[i] = product(u, row_operand<kCols, P, true>(oS, C * kCols, 16 * ct + c, 4 * s + g), p[i]);
                        bb[i] = product(u, row_operand<kCols, 3, true>(wS, C * kCols, 16 * ct + c, 4 * s + g), bb[i]);
                    }
                }
#pragma unroll
                for (int s = 0; s < kCols / 32; ++s) {
                    const int m = m0 + 32 * s + 8 * g;
                    const size_t at = (size_t)unit * D * a.M + (size_t)d * a.M + m;
                    const Eight<float> s0 = load_eight<float>(a.state + at, m < a.M), s1 = load_eight<float>(a.dstate + at, m < a.M);
#pragma unroll
                    for (int e = 0; e < 8; ++e) both = fmaf(s0.get(e), s1.get(e), both);
                    const Parts<3> x0 = cut(f32x4{s0.get(0), s0.get(1), s0.get(2), s0.get(3)}, f32x4{s0.get(4), s0.get(5), s0.get(6), s0.get(7)});
                    const Parts<3> x1 = cut(f32x4{s1.get(0), s1.get(1), s1.get(2), s1.get(3)}, f32x4{s1.get(4), s1.get(5), s1.get(6), s1.get(7)});
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        q1[t] = product(row_operand<kCols, P, true>(oS, C * kCols, 16 * t + c, 4 * s + g), x0, q1[t]);
                        k1[t] = product(row_operand<kCols, 3, true>(wS, C * kCols, 16 * t + c, 4 * s + g), x0, k1[t]);
                        k2[t] = product(row_operand<kCols, 3, true>(uS, C * kCols, 16 * t + c, 4 * s + g), x1, k2[t]);
                    }
                }
            }
            __syncthreads();                                 // U, dV, dO make way for P and B + B^T
#pragma unroll
            for (int i = 0; i < kLowEach; ++i) {
                int n = wave + i * kWaves, ct = 0;
                if (n >= kLow) break;
                while (n > ct) n -= ++ct;
                const int t = 16 * ct + c, s = 16 * n + 4 * g;
                f32x4 pv, bv;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float decay = s + r <= t ? expf((gates[2 * C + t] - gates[2 * C + s + r]) + (gates[3 * C + t] - gates[3 * C + s + r])) : 0.0f;
                    pv[r] = s + r <= t ? a.scale * p[i][r] * decay : 0.0f;
                    bv[r] = s + r < t ? -bb[i][r] * decay : 0.0f;
                }
                const float pq[4] = {pv[0], pv[1], pv[2], pv[3]}, bq[4] = {bv[0], bv[1], bv[2], bv[3]};
                const Split3 ps = split3(pq), bs = split3(bq);
                const u32x2_t parts[2][3] = {{ps.h, ps.m, ps.l}, {bs.h, bs.m, bs.l}};
                const int here = mat_at<C, true>(t, s / 8) + s % 8;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    *reinterpret_cast<u32x2_t *>(pS + k * C * C + here) = parts[0][k];
                    if (n == ct) {                           // on the diagonal both triangles are in one tile
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint16_t e = (uint16_t)(parts[1][k][r / 2] >> (16 * (r & 1)));
                            if (s + r <= t) bS[k * C * C + here + r] = bS[k * C * C + mat_at<C, true>(s + r, t / 8) + t % 8] = e;
                        }
                    } else {
                        *reinterpret_cast<u32x2_t *>(bS + k * C * C + here) = parts[1][k];
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            bS[k * C * C + mat_at<C, true>(s + r, t / 8) + t % 8] = (uint16_t)(parts[1][k][r / 2] >> (16 * (r & 1)));
                    }
                    // the tile right above the diagonal, which products over 32 tokens read
                    if (n == ct && ct % 2 == 0) *reinterpret_cast<u32x2_t *>(pS + k * C * C + mat_at<C, true>(t, (s + 16) / 8) + s % 8) = u32x2_t{0, 0};
                }
            }
            __syncthreads();
            float into = 0.0f;
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 qd, kd, eg, eh;
#pragma unroll
                for (int r = 0; r < 4; ++r) eg[r] = gates[16 * t + 4 * g + r], eh[r] = gates[C + 16 * t + 4 * g + r];
                qd = a.scale * eg * q1[t];
                k2[t] = eh * k2[t];
                kd = k2[t] - eg * k1[t];
#pragma unroll
                for (int s = 0; s < kBlocks; ++s) {
                    const Parts<P> kx = column_operand<D, false, P, true>(kS, C * D, 32 * s, wave, lane);
                    if (s <= t / 2) qd = product(row_operand<C, 3, true>(pS, C * C, 16 * t + c, 4 * s + g), kx, qd);
                    if (s >= t / 2)
                        kd = product(column_operand<C, false, 3, true>(pS, C * C, 32 * s, t, lane), column_operand<D, false, P, true>(qS, C * D, 32 * s, wave, lane), kd);
                    kd = product(row_operand<C, 3, true>(bS, C * C, 16 * t + c, 4 * s + g), kx, kd);
                }
                dq[t] += qd, dk[t] += kd;
                const f32x4 qv = column_values<D, P, true>(qS, C * D, 16 * t + 4 * g, wave, lane).sum(), kv = column_values<D, P, true>(kS, C * D, 16 * t + 4 * g, wave, lane).sum();
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    into = fmaf(kv[r], k2[t][r], into);
                    const float dot = row_sum16(qv[r] * qd[r] - kv[r] * kd[r]);
                    if (c == 0) red[wave][16 * t + 4 * g + r] = dot;
                }
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
    } else {
        for (int i = tid; i < C * per; i += kThreads) {
            const int t = i / per;
            const size_t at = (row0 + t) * a.H + hk * per + i % per;
            if (t0 + t >= a.N) break;
            if (a.dg != nullptr) a.dg[at] = 0.0f;
            a.dbeta[at] = 0.0f;
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = 16 * t + 4 * g + r;
            if (t0 + n >= a.N) continue;
            const size_t at = ((row0 + n) * a.Hk + hk) * D + d;
            store_elem<false>((T *)a.dq + at, n < left ? dq[t][r] : 0.0f);
            store_elem<false>((T *)a.dk + at, n < left ? dk[t][r] : 0.0f);
        }
}
}  // namespace

hipError_t launch_delta_bwd(const DeltaArgs &a, int dtype, hipStream_t s) {
#define LA_STATES(T, D) delta_states_bwd_kernel<T, D><<<head_grid(a), 512, 0, s>>>(a)
    LA_BY_WIDTH(LA_STATES)
    const unsigned units = (unsigned)((long)a.B * a.Hk * a.K);
#define LA_CHUNKS(T, D) delta_chunks_bwd_kernel<T, D><<<units, 4 * D, 0, s>>>(a)
    LA_BY_WIDTH(LA_CHUNKS)
    return hipGetLastError();
}

}  // namespace la
