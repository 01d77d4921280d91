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

template <typename T, int D> __global__ __launch_bounds__(256) void delta_states_bwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks;
    __shared__ uint16_t kS[P * C * D], qS[P * C * D], triS[2 * 3 * Ch::kTri];
    __shared__ float gates[3 * C];
    const uint16_t *zS = triS, *mS = triS + 3 * Ch::kTri;
    int bh, m0;
    if (!head_and_columns(a, bh, m0)) return;
    const int tid = threadIdx.x, lane = tid % kWave, c = lane % 16, g = lane / 16, m = m0 + tid / kWave * 16 + c;
    const bool mine = m < a.M;
    const int b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hk), len = length_of(a, b), chunks = (len + C - 1) / C;
    const size_t seq = (size_t)b * a.N, state = (size_t)bh * D * a.M + m, ldo = (size_t)a.H * a.M;
    f32x4 S[D / 16];                                         // dS'
    load_state<D>(a.dh1 == nullptr || !mine ? nullptr : a.dh1 + state, a.M, g, S);
    Fetch<T, D> next;
    f32x4 v[kTiles];
    const auto load_values = [&](int chunk) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = chunk * C + paired(t, 4 * g + r);
                v[t][r] = mine && n < len ? raw_to_f32((const T *)a.dO + (seq + n) * ldo + (size_t)h * a.M + m) : 0.0f;
            }
    };
    const auto load = [&](int chunk) {
        next.load(a, (long)bh * a.K + chunk, seq + (size_t)chunk * C, len - chunk * C, hk, h, tid);
        load_values(chunk);
    };
    if (mine)                                                // tokens behind the sequence
        for (int n = chunks * C + g; n < a.N; n += 4) store_elem<false>((T *)a.dv + (seq + n) * ldo + (size_t)h * a.M + m, 0.0f);
    if (chunks > 0) load(chunks - 1);
    for (int chunk = chunks - 1; chunk >= 0; --chunk) {
        const long unit = (long)bh * a.K + chunk;
        __syncthreads();
        next.park(kS, qS, triS, gates, tid);
        __syncthreads();
        f32x4 out[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) out[t] = v[t];
        if (chunk > 0) load(chunk - 1);
        if (!mine) continue;
        store_state<D>(a.dstate + (size_t)unit * D * a.M + m, a.M, g, S);
        const auto gate4 = [&](int which, int t) { return *reinterpret_cast<const f32x4 *>(gates + which * C + paired(t, 4 * g)); };
        f32x4 y[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) y[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const Parts<3> x = cut(S[2 * s], S[2 * s + 1]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) y[t] = product(row_operand<D, P>(kS, C * D, paired(t, c), 4 * s + g), x, y[t]);
        }
        Parts<3> x[kBlocks];
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x[s] = cut(out[2 * s], out[2 * s + 1]);        // bf16: the lower parts are zeros
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f32x4 w = {0, 0, 0, 0};
#pragma unroll
            for (int s = t / 2; s < kBlocks; ++s) {
                const Parts<3> mt = column_operand<32, true, 3>(mS, Ch::kTri, tri_row<C>(32 * s, t / 2), t % 2, lane);
                if constexpr (P == 1) w = product(mt, Parts<1>{{x[s].p[0]}}, w);
                else w = product(mt, x[s], w);
            }
            y[t] = a.scale * w + gate4(1, t) * y[t];
        }
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x[s] = cut(gate4(2, 2 * s) * y[2 * s], gate4(2, 2 * s + 1) * y[2 * s + 1]);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f32x4 w = {0, 0, 0, 0};
#pragma unroll
            for (int s = t / 2; s < kBlocks; ++s)
                w = product(column_operand<32, true, 3>(zS, Ch::kTri, tri_row<C>(32 * s, t / 2), t % 2, lane), x[s], w);
            y[t] -= w;
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) a.write[((size_t)unit * C + paired(t, 4 * g + r)) * a.M + m] = y[t][r];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            y[t] = gate4(2, t) * y[t];                       // dV
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = chunk * C + paired(t, 4 * g + r);
                if (n < a.N) store_elem<false>((T *)a.dv + (seq + n) * ldo + (size_t)h * a.M + m, n < len ? y[t][r] : 0.0f);
            }
        }
        const float whole = gates[C - 1];
#pragma unroll
        for (int t = 0; t < D / 16; ++t) S[t] *= whole;
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) {
            const Parts<3> o = cut(a.scale * gate4(0, 2 * s) * out[2 * s], a.scale * gate4(0, 2 * s + 1) * out[2 * s + 1]);
            const Parts<3> w = cut(-gate4(0, 2 * s) * y[2 * s], -gate4(0, 2 * s + 1) * y[2 * s + 1]);
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
                S[t] = product(column_operand<D, true, P>(qS, C * D, 32 * s, t, lane), o, S[t]);
                S[t] = product(column_operand<D, true, P>(kS, C * D, 32 * s, t, lane), w, S[t]);
            }
        }
    }
    if (mine && a.dh0 != nullptr) store_state<D>(a.dh0 + state, a.M, g, S);
}

// Lower parts of a column operand added up again: rows 4g .. + 3 of tile `rows`, column of this lane, in fp32.
template <int COLS, int P> __device__ __forceinline__ f32x4 column_values(const uint16_t *m, int plane, int rows, int tile, int lane) {
    const int q = lane & 15, r = 16 * rows + 4 * (lane >> 4) + (q >> 2), piece = 2 * tile + ((q >> 1) & 1), half = 4 * (q & 1);
    f32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = P - 1; i >= 0; --i) v += widen(read_column(m + i * plane + mat_at<COLS>(r, piece) + half));
    return v;
}

// A workgroup takes one chunk and the heads that share its queries and keys, one after the other, D / 16 waves with 16
// columns of dQ and dK each; the columns of the states 64 at a time.
template <typename T, int D> __global__ __launch_bounds__(4 * D) void delta_chunks_bwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks, kWaves = D / 16, kThreads = 4 * D;
    constexpr int kLow = kTiles * (kTiles + 1) / 2, kLowEach = (kLow + kWaves - 1) / kWaves;
    constexpr int kStage = (6 + P) * C * kCols, kSquares = 6 * C * C, kWork = kStage > kSquares ? kStage : kSquares;
    __shared__ uint16_t kS[P * C * D], qS[P * C * D], work[kWork];
    __shared__ float gates[4 * C], bt[C], miss[C], db[C], red[kWaves][C], ends[kWaves];
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
            park_eight<T>(kS + mat_at<D>(t, piece), C * D, load_eight<T>((const T *)a.k + (row0 + t) * a.ldk + (size_t)hk * D + 8 * piece, t < left));
            park_eight<T>(qS + mat_at<D>(t, piece), C * D, load_eight<T>((const T *)a.q + (row0 + t) * a.ldq + (size_t)hk * D + 8 * piece, t < left));
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
                    const int at = mat_at<kCols>(t, piece);
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
                        const Parts<3> u = row_operand<kCols, 3>(uS, C * kCols, 16 * n + c, 4 * s + g);
                        p[i] = product(u, row_operand<kCols, P>(oS, C * kCols, 16 * ct + c, 4 * s + g), p[i]);
                        bb[i] = product(u, row_operand<kCols, 3>(wS, C * kCols, 16 * ct + c, 4 * s + g), bb[i]);
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
                        q1[t] = product(row_operand<kCols, P>(oS, C * kCols, 16 * t + c, 4 * s + g), x0, q1[t]);
                        k1[t] = product(row_operand<kCols, 3>(wS, C * kCols, 16 * t + c, 4 * s + g), x0, k1[t]);
                        k2[t] = product(row_operand<kCols, 3>(uS, C * kCols, 16 * t + c, 4 * s + g), x1, k2[t]);
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
                const int here = mat_at<C>(t, s / 8) + s % 8;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    *reinterpret_cast<u32x2_t *>(pS + k * C * C + here) = parts[0][k];
                    if (n == ct) {                           // on the diagonal both triangles are in one tile
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const uint16_t e = (uint16_t)(parts[1][k][r / 2] >> (16 * (r & 1)));
                            if (s + r <= t) bS[k * C * C + here + r] = bS[k * C * C + mat_at<C>(s + r, t / 8) + t % 8] = e;
                        }
                    } else {
                        *reinterpret_cast<u32x2_t *>(bS + k * C * C + here) = parts[1][k];
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            bS[k * C * C + mat_at<C>(s + r, t / 8) + t % 8] = (uint16_t)(parts[1][k][r / 2] >> (16 * (r & 1)));
                    }
                    // the tile right above the diagonal, which products over 32 tokens read
                    if (n == ct && ct % 2 == 0) *reinterpret_cast<u32x2_t *>(pS + k * C * C + mat_at<C>(t, (s + 16) / 8) + s % 8) = u32x2_t{0, 0};
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
                    const Parts<P> kx = column_operand<D, false, P>(kS, C * D, 32 * s, wave, lane);
                    if (s <= t / 2) qd = product(row_operand<C, 3>(pS, C * C, 16 * t + c, 4 * s + g), kx, qd);
                    if (s >= t / 2)
                        kd = product(column_operand<C, false, 3>(pS, C * C, 32 * s, t, lane), column_operand<D, false, P>(qS, C * D, 32 * s, wave, lane), kd);
                    kd = product(row_operand<C, 3>(bS, C * C, 16 * t + c, 4 * s + g), kx, kd);
                }
                dq[t] += qd, dk[t] += kd;
                const f32x4 qv = column_values<D, P>(qS, C * D, t, wave, lane), kv = column_values<D, P>(kS, C * D, t, wave, lane);
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
#define LA_STATES(T, D) delta_states_bwd_kernel<T, D><<<head_grid(a), 256, 0, s>>>(a)
    LA_BY_WIDTH(LA_STATES)
    const unsigned units = (unsigned)((long)a.B * a.Hk * a.K);
#define LA_CHUNKS(T, D) delta_chunks_bwd_kernel<T, D><<<units, 4 * D, 0, s>>>(a)
    LA_BY_WIDTH(LA_CHUNKS)
    return hipGetLastError();
}

}  // namespace la
