// Gated delta rule, forward and one token (la_delta_fwd, la_delta_step).
//
//   S_t = e^{g_t} S_{t-1} + beta_t k_t (v_t - e^{g_t} S_{t-1}^T k_t)^T,   o_t = scale S_t^T q_t
//
// Chunks of C tokens.  With G_t the sum of g since the chunk's start, S the state before it, and
//   A_ts = e^{G_t - G_s} k_t . k_s  (s < t),   M_ts = e^{G_t - G_s} q_t . k_s  (s <= t),
// what token t finds missing in the state, u_t = v_t - e^{g_t} S_{t-1}^T k_t, solves u + A beta u = r, r = V - e^G K S:
//   u = r - Z beta r,   Z = (1 + A beta)^-1 A,
//   O = scale (e^G Q S + M beta u),   S' = e^{G_C} S + K^T e^{G_C - G} beta u.
// Z and M do not depend on S: a first launch forms them for all chunks side by side, a second one goes through a sequence's
// chunks.  There a wave has 16 columns of S (and of V, O) for all of its life: K S, Z beta r, M beta u and the update are
// products from the left, each one's result is the next one's operand in the same lanes' registers, and the waves of a
// workgroup share nothing but K, Q, Z and M in LDS.
#include <hip/hip_runtime.h>

#include "la_delta.h"

namespace la {
namespace {

// ---- chunk-local matrices ------------------------------------------------------------------------
// One workgroup a unit: decays, masked products of queries and keys, and the triangular system, column j of Z in lane j.
template <typename T, int D> __global__ __launch_bounds__(256) void delta_local_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kRow = C + 4;
    __shared__ uint16_t kS[P * C * D], qS[P * C * D];
    __shared__ float low[C * kRow];                          // A, strictly lower
    __shared__ float gh[C], gl[C], bt[C];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, c = lane % 16, g = lane / 16;
    const long unit = blockIdx.x;
    const int chunk = (int)(unit % a.K), bh = (int)(unit / a.K), b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hk);
    const int len = length_of(a, b), t0 = chunk * C;
    if (t0 >= len) return;                                   // no later launch reads this unit
    const size_t row0 = (size_t)b * a.N + t0;
    for (int i = tid; i < C * D / 8; i += 256) {
        const int t = i / (D / 8), piece = i % (D / 8);
        const bool live = t0 + t < len;
        const Eight<T> k = load_eight<T>((const T *)a.k + (row0 + t) * a.ldk + (size_t)hk * D + 8 * piece, live);
        const Eight<T> q = load_eight<T>((const T *)a.q + (row0 + t) * a.ldq + (size_t)hk * D + 8 * piece, live);
        park_eight<T>(kS + mat_at<D>(t, piece), C * D, k);
        park_eight<T>(qS + mat_at<D>(t, piece), C * D, q);
    }
    float *gate = a.gate + unit * 4 * C;
    if (wave == 0) {
        const bool live = lane < C && t0 + lane < len;
        const size_t at = (row0 + lane) * a.H + h;
        // sums of many small logarithms, and differences of such sums: fp64, kept as two fp32.  Below -1000 a factor is zero
        // either way, and sums stay finite (a decay to nothing is g = -inf).
        double sum = live && a.g != nullptr ? (double)fmaxf(a.g[at], -1000.0f) : 0.0;
#pragma unroll
        for (int d = 1; d < C; d *= 2) {
            const double from = __shfl_up(sum, d);
            if (lane >= d) sum += from;
        }
        const double whole = __shfl(sum, C - 1);
        if (lane < C) {
            const float hi = (float)sum, lo = (float)(sum - (double)hi);
            gh[lane] = hi, gl[lane] = lo, bt[lane] = live ? a.beta[at] : 0.0f;
            gate[lane] = expf(hi) * (1.0f + lo), gate[C + lane] = expf((float)(whole - sum));
            gate[2 * C + lane] = hi, gate[3 * C + lane] = lo;
        }
    }
    __syncthreads();
    float *zOut = a.tri + unit * 2 * Ch::kTri, *mOut = zOut + Ch::kTri;
    for (int i = wave; i < Ch::kTiles * Ch::kTiles; i += 4) {            // tiles (rt, ct) of 16 x 16
        const int rt = i / Ch::kTiles, ct = i % Ch::kTiles;
        if (ct / 2 > rt / 2) continue;                       // a 32 x 32 block above the diagonal
        f32x4 kk = {0, 0, 0, 0}, qk = {0, 0, 0, 0};
        if (ct <= rt) {
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                const Parts<P> y = row_operand<D, P>(kS, C * D, 16 * ct + c, 4 * s + g);
                kk = product(row_operand<D, P>(kS, C * D, 16 * rt + c, 4 * s + g), y, kk);
                qk = product(row_operand<D, P>(qS, C * D, 16 * rt + c, 4 * s + g), y, qk);
            }
        }
        const int s = 16 * ct + c;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * rt + 4 * g + r;
            const float decay = s <= t ? expf((gh[t] - gh[s]) + (gl[t] - gl[s])) : 0.0f;
            if (ct <= rt) low[t * kRow + s] = s < t ? kk[r] * decay : 0.0f;
            mOut[tri_row<C>(t, ct / 2) * 32 + s % 32] = s <= t ? qk[r] * decay : 0.0f;
        }
    }
    __syncthreads();
    if (wave != 0) return;
    float z[C];
    const int j = lane % C;
#pragma unroll
    for (int r = 0; r < C; ++r) {
        float x = j < r ? low[r * kRow + j] : 0.0f, y = 0.0f;
#pragma unroll
        for (int s = 0; s < r; ++s) {
            const float f = low[r * kRow + s] * bt[s];
            if (s % 2 == 0) x = fmaf(-f, z[s], x);
            else y = fmaf(-f, z[s], y);
        }
        z[r] = x + y;
        if (lane < C && j / 32 <= r / 32) zOut[tri_row<C>(r, j / 32) * 32 + j % 32] = z[r];
    }
}

// ---- through the chunks -----------------------------------------------------------------------------
template <typename T, int D> __global__ __launch_bounds__(256) void delta_fwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks;
    __shared__ uint16_t kS[P * C * D], qS[P * C * D], triS[2 * 3 * Ch::kTri];
    __shared__ float gates[3 * C];
    const uint16_t *zS = triS, *mS = triS + 3 * Ch::kTri;
    int bh, m0;
    if (!head_and_columns(a, bh, m0)) return;
    const int tid = threadIdx.x, lane = tid % kWave, c = lane % 16, g = lane / 16, m = m0 + tid / kWave * 16 + c;
    const bool mine = m < a.M;                               // all of a wave's columns or none (M is a multiple of 16)
    const int b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hk), len = length_of(a, b), chunks = (len + C - 1) / C;
    const size_t seq = (size_t)b * a.N, state = (size_t)bh * D * a.M + m, ldo = (size_t)a.H * a.M;
    f32x4 S[D / 16];
    load_state<D>(a.h0 == nullptr || !mine ? nullptr : a.h0 + state, a.M, g, S);
    Fetch<T, D> next;
    f32x4 v[kTiles];
    const auto load_values = [&](int chunk) {                // a column's elements of the paired rows
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int n = chunk * C + paired(t, 4 * g + r);
                v[t][r] = mine && n < len ? raw_to_f32((const T *)a.v + (seq + n) * a.ldv + (size_t)h * a.M + m) : 0.0f;
            }
    };
    if (chunks > 0) next.load(a, (long)bh * a.K, seq, len, hk, h, tid), load_values(0);
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const long unit = (long)bh * a.K + chunk;
        __syncthreads();                                     // the chunk before has been read
        next.park(kS, qS, triS, gates, tid);
        __syncthreads();
        f32x4 rest[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) rest[t] = v[t];
        if (chunk + 1 < chunks) {
            next.load(a, unit + 1, seq + (size_t)(chunk + 1) * C, len - (chunk + 1) * C, hk, h, tid);
            load_values(chunk + 1);
        }
        if (!mine) continue;
        if (a.state != nullptr) store_state<D>(a.state + (size_t)unit * D * a.M + m, a.M, g, S);
        f32x4 ks[kTiles], qs[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) ks[t] = qs[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const Parts<3> x = cut(S[2 * s], S[2 * s + 1]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                ks[t] = product(row_operand<D, P>(kS, C * D, paired(t, c), 4 * s + g), x, ks[t]);
                qs[t] = product(row_operand<D, P>(qS, C * D, paired(t, c), 4 * s + g), x, qs[t]);
            }
        }
        const auto gate4 = [&](int which, int t) { return *reinterpret_cast<const f32x4 *>(gates + which * C + paired(t, 4 * g)); };
#pragma unroll
        for (int t = 0; t < kTiles; ++t) rest[t] -= gate4(0, t) * ks[t];
        Parts<3> x[kBlocks];
#pragma unroll
        for (int s = 0; s < kBlocks; ++s)
            x[s] = cut(finite(gate4(2, 2 * s) * rest[2 * s]), finite(gate4(2, 2 * s + 1) * rest[2 * s + 1]));
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f32x4 y = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s <= t / 2; ++s)
                y = product(row_operand<32, 3>(zS, Ch::kTri, tri_row<C>(paired(t, c), s), g), x[s], y);
            rest[t] -= y;                                    // what the tokens find missing
        }
        if (a.miss != nullptr) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) a.miss[((size_t)unit * C + paired(t, 4 * g + r)) * a.M + m] = rest[t][r];
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) rest[t] = gate4(2, t) * rest[t];
        if (a.o != nullptr) {
#pragma unroll
            for (int s = 0; s < kBlocks; ++s) x[s] = cut(finite(rest[2 * s]), finite(rest[2 * s + 1]));
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 y = gate4(0, t) * qs[t];
#pragma unroll
                for (int s = 0; s <= t / 2; ++s)
                    y = product(row_operand<32, 3>(mS, Ch::kTri, tri_row<C>(paired(t, c), s), g), x[s], y);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int n = chunk * C + paired(t, 4 * g + r);
                    if (n < a.N) store_elem<false>((T *)a.o + (seq + n) * ldo + (size_t)h * a.M + m, n < len ? a.scale * y[r] : 0.0f);
                }
            }
        }
#pragma unroll
        for (int s = 0; s < kBlocks; ++s)
            x[s] = cut(finite(gate4(1, 2 * s) * rest[2 * s]), finite(gate4(1, 2 * s + 1) * rest[2 * s + 1]));
        const float whole = gates[C - 1];
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
            S[t] *= whole;
#pragma unroll
            for (int s = 0; s < kBlocks; ++s) S[t] = product(column_operand<D, true, P>(kS, C * D, 32 * s, t, lane), x[s], S[t]);
        }
    }
    if (!mine) return;
    if (a.h1 != nullptr) store_state<D>(a.h1 + state, a.M, g, S);
    if (a.o != nullptr)
        for (int n = chunks * C + g; n < a.N; n += 4) store_elem<false>((T *)a.o + (seq + n) * ldo + (size_t)h * a.M + m, 0.0f);
}

// ---- one token ------------------------------------------------------------------------------------------
// A workgroup has 64 columns of a head's state, 16 lanes a row (four columns each), 16 rows at a time: the state is read
// once and written once.  k . S and q . S are formed together, o = e^g q . S + (q . k) beta u, so that the sums over the rows meet once.
template <typename T, int D> __global__ __launch_bounds__(256) void delta_step_kernel(const DeltaArgs a, float *h) {
    constexpr int kRows = D / 16;
    __shared__ f32x4 red[4][2][16];
    __shared__ float dots[4];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, l = tid % 16, part = tid / 16;
    const int blocks = (a.M + kCols - 1) / kCols, bh = blockIdx.x / blocks, m = blockIdx.x % blocks * kCols + 4 * l;
    const int b = bh / a.H, head = bh % a.H, hk = head / (a.H / a.Hk);
    const bool mine = m < a.M;
    float *S = h + (size_t)bh * D * a.M + m;
    f32x4 s[kRows];
    float k[kRows], q[kRows];
    const T *kp = (const T *)a.k + ((size_t)b * a.Hk + hk) * D, *qp = (const T *)a.q + ((size_t)b * a.Hk + hk) * D;
#pragma unroll
    for (int i = 0; i < kRows; ++i) s[i] = mine ? *reinterpret_cast<const f32x4 *>(S + (size_t)(16 * i + part) * a.M) : f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kRows; ++i) k[i] = raw_to_f32(kp + 16 * i + part), q[i] = raw_to_f32(qp + 16 * i + part);
    f32x4 v = {0, 0, 0, 0};
    if (mine)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = raw_to_f32((const T *)a.v + (size_t)bh * a.M + m + i);
    const float decay = a.g != nullptr ? expf(a.g[bh]) : 1.0f, beta = a.beta[bh];
    f32x4 ks = {0, 0, 0, 0}, qs = {0, 0, 0, 0};
    float qk = 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        s[i] *= decay;
        ks += k[i] * s[i], qs += q[i] * s[i];
        qk = fmaf(q[i], k[i], qk);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) ks[i] = add_halves(add_rows(ks[i])), qs[i] = add_halves(add_rows(qs[i]));
    qk = add_halves(add_rows(qk));
    if (lane < 16) red[wave][0][l] = ks, red[wave][1][l] = qs;
    if (lane == 0) dots[wave] = qk;
    __syncthreads();
    ks = (red[0][0][l] + red[1][0][l]) + (red[2][0][l] + red[3][0][l]);
    qs = (red[0][1][l] + red[1][1][l]) + (red[2][1][l] + red[3][1][l]);
    qk = (dots[0] + dots[1]) + (dots[2] + dots[3]);
    if (!mine) return;
    const f32x4 write = beta * (v - ks);
#pragma unroll
    for (int i = 0; i < kRows; ++i) *reinterpret_cast<f32x4 *>(S + (size_t)(16 * i + part) * a.M) = s[i] + k[i] * write;
    if (part == 0) {
        const f32x4 y = a.scale * (qs + qk * write);
#pragma unroll
        for (int i = 0; i < 4; ++i) store_elem<false>((T *)a.o + (size_t)bh * a.M + m + i, y[i]);
    }
}
}  // namespace

hipError_t launch_delta_fwd(const DeltaArgs &a, int dtype, hipStream_t s) {
    const unsigned units = (unsigned)((long)a.B * a.H * a.K);
#define LA_LOCAL(T, D) delta_local_kernel<T, D><<<units, 256, 0, s>>>(a)
    LA_BY_WIDTH(LA_LOCAL)
#define LA_PASS(T, D) delta_fwd_kernel<T, D><<<head_grid(a), 256, 0, s>>>(a)
    LA_BY_WIDTH(LA_PASS)
    return hipGetLastError();
}

hipError_t launch_delta_step(const DeltaArgs &a, float *h, int dtype, hipStream_t s) {
    const unsigned grid = (unsigned)(a.B * a.H * ((a.M + kCols - 1) / kCols));
#define LA_STEP(T, D) delta_step_kernel<T, D><<<grid, 256, 0, s>>>(a, h)
    LA_BY_WIDTH(LA_STEP)
    return hipGetLastError();
}

}  // namespace la
