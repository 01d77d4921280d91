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
// Decays, masked products of queries and keys, and the triangular system (1 + A beta) Z = A by blocks
// of 16.  The inverse of the diagonal blocks comes by substitution, one block in each lane group and one column a lane; then a
// wave has a block column of Z, Z_ij = (1 + A beta)_ii^-1 (A_ij - sum_k (A beta)_ik Z_kj), whose products feed each other in
// registers.  All in fp32 (v_mfma_f32_16x16x4: lane (c, g) supplies elements 4g + q of its row c, register q of a result is that
// of the next operand).
constexpr int tri_stride(int C) { return C + 4; }            // floats between rows: 16 rows' 16-byte reads meet all banks
__device__ __forceinline__ f32x4 times(f32x4 rows, f32x4 columns, f32x4 acc) {
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = mfma16(rows[q], columns[q], acc);
    return acc;
}
// block (i, j) of a matrix as the left operand, and as the right one
template <int C> __device__ __forceinline__ f32x4 block_rows(const float *m, int i, int j, int c, int g) {
    return *reinterpret_cast<const f32x4 *>(m + (16 * i + c) * tri_stride(C) + 16 * j + 4 * g);
}
template <int C> __device__ __forceinline__ f32x4 block_columns(const float *m, int i, int j, int c, int g) {
    f32x4 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = m[(16 * i + 4 * g + q) * tri_stride(C) + 16 * j + c];
    return v;
}
// of the lane n places before in its row of 16 (zero without one), and of one lane
template <int n> __device__ __forceinline__ double lane_before(double v) {
    const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
    return __builtin_bit_cast(double, u32x2_t{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], 0x110 + n, 0xf, 0xf, true),
                                              (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], 0x110 + n, 0xf, 0xf, true)});
}
__device__ __forceinline__ double value_of(double v, int lane) {
    const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
    return __builtin_bit_cast(double, u32x2_t{(uint32_t)__builtin_amdgcn_readlane((int)w[0], lane), (uint32_t)__builtin_amdgcn_readlane((int)w[1], lane)});
}
// One wave, a token a lane: G as hi + lo, e^G and e^{G_C - G}.  Sums of many small logarithms, and differences of such sums: fp64,
// kept as two fp32.  Below -1000 a factor is zero either way, and sums stay finite (a decay to nothing is g = -inf).
template <int C> __device__ __forceinline__ void decays(float gate_in, int g, float &hi, float &lo, float &since, float &rest) {
    double sum = (double)(gate_in < -1000.0f ? -1000.0f : gate_in);      // a NaN stays one
    sum += lane_before<1>(sum), sum += lane_before<2>(sum), sum += lane_before<4>(sum), sum += lane_before<8>(sum);
    double before = 0.0;                                     // and over the rows of 16 lanes
#pragma unroll
    for (int r = 1; r < C / 16; ++r) before += g >= r ? value_of(sum, 16 * r - 1) : 0.0;
    sum += before;
    const double whole = value_of(sum, C - 1);
    hi = (float)sum, lo = (float)(sum - (double)hi);
    since = expf(hi) * (1.0f + lo), rest = expf((float)(whole - sum));
}
// The tiles of 16 x 16 on and below a chunk's diagonal, dealt to four waves; where a wave has fewer, the last one again, not put out.
template <int C> struct LowTiles {
    static constexpr int kTiles = C / 16, kLow = kTiles * (kTiles + 1) / 2, kEach = (kLow + 3) / 4;
    int row[kEach], col[kEach], wave;
    __device__ __forceinline__ explicit LowTiles(int w) : wave(w) {
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            const int i = wave + 4 * n < kLow ? wave + 4 * n : kLow - 1;
            row[n] = i < 1 ? 0 : i < 3 ? 1 : i < 6 ? 2 : 3, col[n] = i - row[n] * (row[n] + 1) / 2;
        }
    }
    __device__ __forceinline__ bool mine(int n) const { return wave + 4 * n < kLow; }
};
// A into LDS, M's tiles into registers
template <typename T, int D, bool kPlain> __device__ __forceinline__ void masked_products(const uint16_t *kS, const uint16_t *qS, const float *gh, const float *gl, float *low,
                                                                                         const LowTiles<Chunk<T>::C> &at, f32x4 (&M)[LowTiles<Chunk<T>::C>::kEach], int c, int g) {
    constexpr int C = Chunk<T>::C, P = Chunk<T>::P, kEach = LowTiles<C>::kEach;
    f32x4 kk[kEach];
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
        kk[n] = M[n] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const Parts<P> y = row_operand<D, P, kPlain>(kS, C * D, 16 * at.col[n] + c, 4 * s + g);
            kk[n] = product(row_operand<D, P, kPlain>(kS, C * D, 16 * at.row[n] + c, 4 * s + g), y, kk[n]);
            M[n] = product(row_operand<D, P, kPlain>(qS, C * D, 16 * at.row[n] + c, 4 * s + g), y, M[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < kEach; ++n) {
        const int s = 16 * at.col[n] + c, first = 16 * at.row[n] + 4 * g;
        const f32x4 hi = *reinterpret_cast<const f32x4 *>(gh + first) - gh[s], lo = *reinterpret_cast<const f32x4 *>(gl + first) - gl[s];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float decay = s <= first + r ? decay_of(hi[r], lo[r]) : 0.0f;
            kk[n][r] = s < first + r ? kk[n][r] * decay : 0.0f;
            M[n][r] = s <= first + r ? M[n][r] * decay : 0.0f;
        }
        if (at.mine(n))
#pragma unroll
            for (int r = 0; r < 4; ++r) low[(first + r) * tri_stride(C) + s] = kk[n][r];
    }
}
// Z's block column `wave` into registers, from A and beta in LDS; inv: room for as much again.  All four waves; a barrier inside.
template <int C> __device__ __forceinline__ void solve(const float *low, float *inv, const float *bt, int wave, int c, int g, f32x4 (&z)[C / 16]) {
    constexpr int kTiles = C / 16;
    if (wave == 0 && g < kTiles) {
        f32x4 f[16][4];
#pragma unroll
        for (int r = 1; r < 16; ++r)
#pragma unroll
            for (int q = 0; 4 * q < r; ++q) f[r][q] = *reinterpret_cast<const f32x4 *>(low + (16 * g + r) * tri_stride(C) + 16 * g + 4 * q);
        float x[16], y[16];                                  // column c of block (g, g), and beta times it
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float v = r == c ? 1.0f : 0.0f, u = 0.0f;
#pragma unroll
            for (int s = 0; s < r; ++s) {
                if (s % 2 == 0) v = fmaf(-f[r][s / 4][s % 4], y[s], v);
                else u = fmaf(-f[r][s / 4][s % 4], y[s], u);
            }
            x[r] = v + u, y[r] = bt[16 * g + r] * x[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) inv[(16 * g + r) * tri_stride(C) + 16 * g + c] = x[r];
    }
    f32x4 ab[kTiles][kTiles];                                // z: what is left of A; -(A beta)
    const int j = wave;
    if (j < kTiles) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            if (i >= j) z[i] = block_columns<C>(low, i, j, c, g);
#pragma unroll
            for (int k = 0; k < i; ++k)
                if (k >= j) ab[i][k] = -block_rows<C>(low, i, k, c, g) * *reinterpret_cast<const f32x4 *>(bt + 16 * k + 4 * g);
        }
    }
    __syncthreads();
    if (j < kTiles) {
#pragma unroll
        for (int k = 0; k < kTiles; ++k) {
            if (k < j) continue;
            z[k] = times(block_rows<C>(inv, k, k, c, g), finite(z[k]), f32x4{0, 0, 0, 0});
            const f32x4 y = finite(z[k]);
#pragma unroll
            for (int i = k + 1; i < kTiles; ++i) z[i] = times(ab[i][k], y, z[i]);
        }
    }
}
// Both matrices element by element: put(matrix, row of it, column of 32, value), M = 1; with the zeros right of a diagonal tile that
// lie in the same 32 x 32 block.
template <int C, typename Put> __device__ __forceinline__ void put_out_m(const LowTiles<C> &at, const f32x4 (&M)[LowTiles<C>::kEach], int c, int g, Put put) {
#pragma unroll
    for (int n = 0; n < LowTiles<C>::kEach; ++n) {
        if (!at.mine(n)) break;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = tri_row<C>(16 * at.row[n] + 4 * g + r, at.col[n] / 2);
            put(1, row, (16 * at.col[n] + c) % 32, M[n][r]);
            if (at.row[n] == at.col[n] && at.row[n] % 2 == 0) put(1, row, 16 + c, 0.0f);
        }
    }
}
template <int C, typename Put> __device__ __forceinline__ void put_out_z(int j, const f32x4 (&z)[C / 16], int c, int g, Put put) {
    if (j >= C / 16) return;
#pragma unroll
    for (int i = 0; i < C / 16; ++i) {
        if (i < j) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = tri_row<C>(16 * i + 4 * g + r, j / 2);
            put(0, row, (16 * j + c) % 32, z[i][r]);
            if (i == j && i % 2 == 0) put(0, row, 16 + c, 0.0f);
        }
    }
}
// One workgroup a unit.  Every step waits for the one before, so what counts is how many workgroups a compute unit holds: three of 128
// columns; else four in bf16, five of 64 columns and eight of 32 in fp32.  8 x 2048 x 16 heads of 128 bf16: 63 us, 3.8 TB/s of tokens and matrices.
template <typename T, int D> __global__ __launch_bounds__(256, D == 128 ? (sizeof(T) == 2 ? 3 : 2) : 4) void delta_local_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTokens = 2 * P * C * D * (int)sizeof(uint16_t), kTri = C * tri_stride(C) * (int)sizeof(float);
    __shared__ alignas(16) char space[kTokens > kTri ? kTokens : kTri];
    __shared__ alignas(16) float low[C * tri_stride(C)];     // A, zeros on the diagonal and above
    __shared__ alignas(16) float gh[C], gl[C], bt[C];
    uint16_t *kS = reinterpret_cast<uint16_t *>(space), *qS = kS + P * C * D;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), c = lane % 16, g = lane / 16;
    const unsigned unit = blockIdx.x;                        // below 2^23
    const int chunk = (int)(unit % (unsigned)a.K), bh = (int)(unit / (unsigned)a.K), b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hk);
    const int len = length_of(a, b), t0 = chunk * C, left = len - t0;
    if (left <= 0) return;                                   // no later launch reads this unit
    const size_t row0 = (size_t)b * a.N + t0;
    const Range kr = range_of((const T *)a.k + row0 * a.ldk + (size_t)hk * D, left < C ? left : C, a.ldk, D);
    const Range qr = range_of((const T *)a.q + row0 * a.ldq + (size_t)hk * D, left < C ? left : C, a.ldq, D);
    const size_t at = (row0 + lane) * a.H + h;
    const bool live = wave == 0 && lane < C && lane < left;
    const float gate_in = live && a.g != nullptr ? a.g[at] : 0.0f, beta_in = live ? a.beta[at] : 0.0f;
    constexpr int kEach = (C * D / 8 + 255) / 256;
    Eight<T> kq[kEach][2];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
        kq[j][0] = load_eight<T>(kr, (t * (int)a.ldk + 8 * piece) * (int)sizeof(T));
        kq[j][1] = load_eight<T>(qr, (t * (int)a.ldq + 8 * piece) * (int)sizeof(T));
    }
    float *gate = a.gate + (size_t)unit * 4 * C;
    if (wave == 0) {
        float hi, lo, since, rest;
        decays<C>(gate_in, g, hi, lo, since, rest);
        if (lane < C) {
            gh[lane] = hi, gl[lane] = lo, bt[lane] = beta_in;
            gate[lane] = since, gate[C + lane] = rest, gate[2 * C + lane] = hi, gate[3 * C + lane] = lo;
        }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
        if (C * D / 8 % 256 != 0 && i >= C * D / 8) break;
        park_eight<T>(kS + mat_at<D, true>(t, piece), C * D, kq[j][0]);
        park_eight<T>(qS + mat_at<D, true>(t, piece), C * D, kq[j][1]);
    }
    __syncthreads();
    float *out = a.tri + (size_t)unit * 2 * Ch::kTri;
    const auto put = [&](int matrix, int row, int column, float v) { out[matrix * Ch::kTri + row * 32 + column] = v; };
    const LowTiles<C> tiles(wave);
    f32x4 M[LowTiles<C>::kEach], z[C / 16];
    masked_products<T, D, true>(kS, qS, gh, gl, low, tiles, M, c, g);
    put_out_m<C>(tiles, M, c, g, put);
    __syncthreads();                                         // K and Q make way for the inverses
    solve<C>(low, reinterpret_cast<float *>(space), bt, wave, c, g, z);
    put_out_z<C>(wave, z, c, g, put);
}
// All that a sequence of one chunk needs, in the place that a pass reads it from.  A and the inverses lie where Z and M come to be.
template <typename T, int D> __device__ __forceinline__ void only_chunk(Chunked<T, D> &to, float *gh, float *gl, const DeltaArgs &a, const Task &task, int tid) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, kTok = C * D / 8, kTokEach = (kTok + 255) / 256, kValEach = C * kCols / 8 / 256;
    static_assert(C * tri_stride(C) * sizeof(float) <= sizeof(to.z), "room for a matrix of fp32");
    const int lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), c = lane % 16, g = lane / 16, hk = task.h / (a.H / a.Hk), rows = task.len < C ? task.len : C;
    const size_t row0 = (size_t)task.b * a.N, at = (row0 + lane) * a.H + task.h;
    const Range kr = range_of((const T *)a.k + row0 * a.ldk + (size_t)hk * D, rows, a.ldk, D), qr = range_of((const T *)a.q + row0 * a.ldq + (size_t)hk * D, rows, a.ldq, D);
    const Range vr = range_of((const T *)a.v + row0 * a.ldv + (size_t)task.h * a.M + task.m0, rows, a.ldv, task.cols);
    const bool live = wave == 0 && lane < rows;
    const float gate_in = live && a.g != nullptr ? a.g[at] : 0.0f, beta_in = live ? a.beta[at] : 0.0f;
    Eight<T> kq[kTokEach][2], v[kValEach];
#pragma unroll
    for (int j = 0; j < kTokEach; ++j) {
        const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
        kq[j][0] = load_eight<T>(kr, (t * (int)a.ldk + 8 * piece) * (int)sizeof(T));
        kq[j][1] = load_eight<T>(qr, (t * (int)a.ldq + 8 * piece) * (int)sizeof(T));
    }
#pragma unroll
    for (int j = 0; j < kValEach; ++j) {
        const int i = tid + 256 * j, t = i / 8, piece = i % 8;
        v[j] = load_eight<T>(vr, 8 * piece < task.cols ? (t * (int)a.ldv + 8 * piece) * (int)sizeof(T) : 0x7fffff00);
    }
    if (wave == 0) {
        float hi, lo, since, rest;
        decays<C>(gate_in, g, hi, lo, since, rest);
        if (lane < C) gh[lane] = hi, gl[lane] = lo, to.gates[lane] = since, to.gates[C + lane] = rest, to.gates[2 * C + lane] = beta_in;
    }
#pragma unroll
    for (int j = 0; j < kTokEach; ++j) {
        const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
        if (kTok % 256 != 0 && i >= kTok) break;
        park_eight<T>(to.k + mat_at<D>(t, piece), C * D, kq[j][0]);
        park_eight<T>(to.q + mat_at<D>(t, piece), C * D, kq[j][1]);
    }
#pragma unroll
    for (int j = 0; j < kValEach; ++j) {
        const int i = tid + 256 * j;
        park_columns<T>(to.v + mat_at<kCols>(i / 8, i % 8), C * kCols, v[j]);
    }
    __syncthreads();
    float *low = reinterpret_cast<float *>(to.z), *inv = reinterpret_cast<float *>(to.m);
    const LowTiles<C> tiles(wave);
    f32x4 M[LowTiles<C>::kEach], z[C / 16];
    masked_products<T, D, false>(to.k, to.q, gh, gl, low, tiles, M, c, g);
    __syncthreads();
    solve<C>(low, inv, to.gates + 2 * C, wave, c, g, z);
    __syncthreads();                                         // both have been read
    const auto put = [&](int matrix, int row, int column, float x) {
        const float pair[4] = {x, 0.0f, 0.0f, 0.0f};
        const Split3 p = split3(pair);
        uint16_t *m = (matrix ? to.m : to.z) + mat_at<32>(row, column / 8) + column % 8;
        m[0] = (uint16_t)p.h[0], m[Ch::kTri] = (uint16_t)p.m[0], m[2 * Ch::kTri] = (uint16_t)p.l[0];
    };
    put_out_m<C>(tiles, M, c, g, put);
    put_out_z<C>(wave, z, c, g, put);
}

// A token that writes what is no finite number spoils its column: its output, those behind it and the state are NaN, as token by token.
// (What meets masked zeros is made finite, which would hide it.)  Here the outputs, behind a branch that is else not taken.
template <int C, int N> __device__ __forceinline__ void spoil_outputs(const f32x4 (&written)[N], f32x4 (&out)[N], int g) {
    int from = C;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (written[t][r] * 0.0f != 0.0f) from = min(from, paired(t, 4 * g + r));
    from = min(from, __shfl_xor(from, 16));                  // over the lanes of a column
    from = min(from, __shfl_xor(from, 32));
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) out[t][r] = paired(t, 4 * g + r) >= from ? __builtin_nanf("") : out[t][r];
}

// All products take three parts a value, also Q S and M beta u for outputs in bf16: they may cancel, and two parts (2^-16) of a state of 2^17
// were up to 1 off, where three are 2^-6 (with two, and without the test above: training step of 8 x 2048 x 16 heads of 128 bf16 733 us, now 743;
// one prompt of 32768 tokens 650, now 673; training step of 8 x 784 x 8 heads of 32 bf16 98, now 103).
// A chunk is one long chain of products with one working wave a SIMD, so the operands of each product are read from LDS while
// the one before runs, products that the chain does not wait for run beside the cutting of values, and the loop's one branch is
// that of spoiled columns.  Of 128 x 128 bf16 a chunk is 216 matrix instructions of 16 cycles, some 520 vector ones of 4, and waits: 3.5 us;
// 8 x 2048 x 16 heads with what the backward needs, 470 MB written: 228 us, 3.3 TB/s.  (16 columns a wave: a state of 128 rows and its parts
// are 80 registers; 64 a workgroup: two buffers of a chunk are 157 KB of LDS.)
// Sequences of one chunk at most have nothing to fetch ahead: the working waves fetch it themselves (kAlone), two workgroups of half
// the threads and LDS a compute unit, or form its matrices too (kAll), with no launch to wait for.  64 x 33 tokens, 8 heads of 64 bf16:
// 24.1 us as a pass, 20.0 alone, 17.1 all in one.  Every 64 columns form the matrices again: with two such blocks no slower (1024 heads
// of 64 tokens and 128 x 128: 74 and 75 us), with four (64 x 256) 100 us, 83 alone and 118 as a pass.
enum OneChunk { kPass, kAlone, kAll };
template <typename T, int D, PassKind kKind, bool kKeep, OneChunk kHow = kPass> __global__ __launch_bounds__(kHow != kPass ? 256 : 512, kKind == kTransitions && two_lean(sizeof(T), D) ? 4 : 2) void delta_fwd_kernel(const DeltaArgs a) {
    using Ch = Chunk<T>;
    constexpr int C = Ch::C, P = Ch::P, kTiles = Ch::kTiles, kBlocks = Ch::kBlocks, kSteps = D / 32;
    constexpr bool kOutputs = kKind == kWhole, kOne = kHow != kPass;
    __shared__ Chunked<T, D, !kOutputs> buffers[kOne ? 1 : 2];
    Task task;
    if (!task_of<kKind, false>(a, C, D, task)) return;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), c = lane % 16, g = lane / 16, m = task.m0 + wave * 16 + c;
    const int h = task.h, len = task.len, count = task.count, ldo = a.H * a.M;
    const size_t seq = (size_t)task.b * a.N, state = (size_t)task.bh * D * a.M, piece = (size_t)task.bh * a.pieces + task.piece;
    if constexpr (kHow == kAlone) {
        if (count > 0) fetch_only<T, D>(buffers[0], a, task, (const T *)a.v, a.ldv, tid);
    } else if constexpr (kHow == kAll) {
        __shared__ alignas(16) float gh[C], gl[C];
        if (count > 0) only_chunk<T, D>(buffers[0], gh, gl, a, task, tid);
    } else if (wave >= 4) {
        fetch_chunks<T, D, !kOutputs, false>(buffers, a, task, (const T *)a.v, a.ldv, tid - 256);
        return;
    }
    if (wave * 16 >= task.cols) {                            // no columns (M is a multiple of 16)
        if (count > 0) __syncthreads();
        if constexpr (!kOne)
            for (int i = 0; i < count; ++i) __syncthreads();
        return;
    }
    f32x4 S[D / 16];
    const float *from = task.start ? (a.h0 == nullptr ? nullptr : a.h0 + state) : kOutputs ? a.piece_state + piece * D * a.M : nullptr;
    load_state<D>(from, m, a.M, g, S);
    if (kKind == kTransitions && task.unit) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = paired(t, 4 * g + r) == m ? 1.0f : 0.0f;
    }
    loads_done();
    Parts<3> sp[kSteps];                                     // the state as an operand
#pragma unroll
    for (int s = 0; s < kSteps; ++s) sp[s] = cut(S[2 * s], S[2 * s + 1]);
    const int most = a.o == nullptr ? 0 : C;                 // no outputs are asked for: stores go nowhere
    if (count > 0) __syncthreads();
    for (int i = 0; i < count; ++i) {
        const int chunk = task.first + i;
        const long unit = (long)task.bh * a.K + chunk;
        const size_t row0 = seq + (size_t)chunk * C;
        const int left = len - chunk * C;
        const Chunked<T, D, !kOutputs> &in = buffers[kOne ? 0 : i & 1];
        const auto gate4 = [&](int which, int t) { return *reinterpret_cast<const f32x4 *>(in.gates + which * C + paired(t, 4 * g)); };
        const auto rows = [&](const uint16_t *mat, int s, Parts<P> (&f)[kTiles]) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) f[t] = row_operand<D, P>(mat, C * D, paired(t, c), 4 * s + g);
        };
        f32x4 ks[kTiles], qs[kTiles], rest[kTiles], since[kTiles], strength[kTiles];
        Raw4<P> v[kTiles];
        Parts<P> f[2][kTiles];
        // K S; what comes with it is on its way meanwhile
        rows(in.k, 0, f[0]);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) ks[t] = qs[t] = f32x4{0, 0, 0, 0};
        if constexpr (kKeep) store_state<D>(a.state + (size_t)unit * D * a.M, m - c, a.M, lane, S);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if (s + 1 < kSteps) rows(in.k, s + 1, f[(s + 1) % 2]);
            else {
                if (kOutputs) rows(in.q, 0, f[kSteps % 2]);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    v[t] = column_values<kCols, P>(in.v, C * kCols, paired(t, 4 * g), wave, lane);
                    since[t] = gate4(0, t), strength[t] = gate4(2, t);
                }
            }
            in_this_order<D>();
            products(f[s % 2], sp[s], ks);
        }
        in_this_order<D>();
        // Q S beside what the tokens miss of the state before the chunk
        Parts<3> x[kBlocks], zf[kTiles][kBlocks];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) rest[t] = v[t].sum() - since[t] * ks[t];
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x[s] = cut(finite(strength[2 * s] * rest[2 * s]), finite(strength[2 * s + 1] * rest[2 * s + 1]));
        if constexpr (kOutputs) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                if (s + 1 < kSteps) rows(in.q, s + 1, f[(kSteps + s + 1) % 2]);
                products(f[(kSteps + s) % 2], sp[s], qs);
            }
            side_by_side<D, kSteps * kTiles * (P == 1 ? 3 : 6)>();
        }
        in_this_order<D>();
        // ... and of what the chunk's earlier tokens write
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
#pragma unroll
            for (int t = 2 * i; t < kTiles; ++t) zf[t][i] = row_operand<32, 3>(in.z, Ch::kTri, tri_row<C>(paired(t, c), i), g);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) ks[t] = f32x4{0, 0, 0, 0};
        lower_products(zf, x, ks);
        in_this_order<D>();
        Parts<3> mf[kTiles][kBlocks], u[kBlocks];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            qs[t] *= since[t];
            if constexpr (kOutputs)
#pragma unroll
                for (int i = 0; i <= t / 2; ++i) mf[t][i] = row_operand<32, 3>(in.m, Ch::kTri, tri_row<C>(paired(t, c), i), g);
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) rest[t] -= ks[t];
        if constexpr (kKeep) {
            const Range r = range_of(a.miss + (size_t)unit * C * a.M, C, a.M, a.M);
            const int l = here(lane);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) store_tile<float>(r, paired(t, 4 * (l / 16)), task.m0 + wave * 16, a.M, rest[t], l);
        }
        float spoiled = 0.0f;                                // NaN where a token writes what is no finite number
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            rest[t] *= strength[t];
#pragma unroll
            for (int r = 0; r < 4; ++r) spoiled = fmaf(rest[t][r], 0.0f, spoiled);
        }
        if (kOutputs && __any(spoiled != 0.0f)) spoil_outputs<C>(rest, qs, g);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) rest[t] = finite(rest[t]);
        if constexpr (kOutputs)
#pragma unroll
            for (int s = 0; s < kBlocks; ++s) u[s] = cut(rest[2 * s], rest[2 * s + 1]);
        constexpr int kGroup = 4 < D / 16 ? 4 : D / 16, kGroups = D / 16 / kGroup;      // tiles of the state at a time
        Parts<P> kt[2][kGroup];
        const auto columns = [&](int n) {                    // n counts (group, block)
#pragma unroll
            for (int t = 0; t < kGroup; ++t) kt[n % 2][t] = column_operand<D, true, P>(in.k, C * D, 32 * (n % kBlocks), n / kBlocks * kGroup + t, lane);
        };
        in_this_order<D>();
        columns(0);
#pragma unroll
        for (int t = 0; t < kTiles; ++t) since[t] = gate4(1, t);
        if constexpr (kOutputs) lower_products(mf, u, qs);
#pragma unroll
        for (int s = 0; s < kBlocks; ++s) x[s] = cut(finite(since[2 * s] * rest[2 * s]), finite(since[2 * s + 1] * rest[2 * s + 1]));
        const float whole = in.gates[C - 1];
        spoiled = add_halves(add_rows(spoiled));             // of the lanes of a column
#pragma unroll
        for (int t = 0; t < D / 16; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = fmaf(S[t][r], whole, spoiled);
        if (kOutputs) side_by_side<D, (kTiles == 4 ? 6 : 2) * 6>();
        in_this_order<D>();
        const Range r = range_of((T *)a.o + row0 * ldo + (size_t)h * a.M, left < most ? left : most, ldo, a.M);
#pragma unroll
        for (int n = 0; n < kGroups * kBlocks; ++n) {
            if (n + 1 < kGroups * kBlocks) columns(n + 1);
            f32x4 part[kGroup];
#pragma unroll
            for (int t = 0; t < kGroup; ++t) part[t] = S[n / kBlocks * kGroup + t];
            products(kt[n % 2], x[n % kBlocks], part);
#pragma unroll
            for (int t = 0; t < kGroup; ++t) S[n / kBlocks * kGroup + t] = part[t];
            if (kOutputs && n == 0) {
#pragma unroll
                for (int t = 0; t < kTiles; ++t) store_tile<T>(r, paired(t, 4 * g), m - c, ldo, a.scale * qs[t], lane);
            }
            if (n % kBlocks == 0 && n > 0) {                 // the group before is complete
#pragma unroll
                for (int s = 0; s < kGroup / 2; ++s) {
                    const int i = (n / kBlocks - 1) * kGroup / 2 + s;
                    sp[i] = cut(S[2 * i], S[2 * i + 1]);
                }
            }
            if (n == 0 || n % kBlocks == 0) side_by_side<D, kGroup * (P == 1 ? 3 : 6)>();
            in_this_order<D>();
        }
#pragma unroll
        for (int i = (kGroups - 1) * kGroup / 2; i < kSteps; ++i) sp[i] = cut(S[2 * i], S[2 * i + 1]);
        if constexpr (kOne) break;
        else __syncthreads();
    }
    if constexpr (kOutputs) {
        if (!task.end) return;
        if (a.h1 != nullptr) store_state<D>(a.h1 + state, m - c, a.M, lane, S);
        if (a.o != nullptr)                                  // tokens behind the sequence
            for (int n = len + g; n < a.N; n += 4) store_elem<false>((T *)a.o + (seq + n) * ldo + (size_t)h * a.M + m, 0.0f);
    } else if (task.unit) {
        store_state<D>(a.transition + piece * D * D, m - c, D, lane, S);
    } else {
        store_state<D>(a.piece_state + (piece + 1) * D * a.M, m - c, a.M, lane, S);
    }
}

// ---- from piece to piece -----------------------------------------------------------------------------
// Forwards S_{j+1} = F_j S_j + (what piece j leaves of a zero state), j = 1 .. last - 1; backwards E_{j-1} = F_j^T E_j + .., j = last - 1
// .. 1.  kJoin columns a workgroup; a wave has some rows of the transitions F, on their way a piece ahead, and all of the
// columns, which the waves hand each other through LDS.  A piece waits for the one before, so few columns: with 64, 6.5 us a piece of
// 16 heads of 128 x 128 and 2.6 of 64 x 64, with 16, 4.9 and 1.5.
constexpr int kJoin = 16;
template <int D, bool kBack> __global__ __launch_bounds__(256) void delta_join_kernel(const DeltaArgs a, float *states, int C) {
    constexpr int kEach = D <= 64 ? 1 : D / 64, kSteps = D / 32;
    __shared__ alignas(16) uint16_t sS[2][3 * kJoin * D];
    const int blocks = (a.M + kJoin - 1) / kJoin, bh = blockIdx.x / blocks, m0 = blockIdx.x % blocks * kJoin;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), c = lane % 16, g = lane / 16;
    const int cols = a.M - m0 < kJoin ? a.M - m0 : kJoin, chunks = (length_of(a, bh / a.H) + C - 1) / C, last = chunks > 0 ? (chunks - 1) / a.length : 0;
    const bool mine = wave * kEach * 16 < D;                 // of 32 rows two waves have none
    float *state = states + (size_t)bh * a.pieces * D * a.M;
    const float *transition = a.transition + (size_t)bh * a.pieces * D * D;
    const int count = last - 1;
    if (count <= 0) return;
    const auto from = [&](int i) { return kBack ? last - 1 - i : 1 + i; };              // the i-th piece, and the state it starts from
    f32x4 rows[kEach][kSteps][2];
    const auto load_rows = [&](int piece) {
        const float *f = transition + (size_t)piece * D * D;
#pragma unroll
        for (int x = 0; x < kEach; ++x)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int row = mine ? 16 * (wave * kEach + x) + c : c, at = 32 * s + 8 * g;
#pragma unroll
                for (int i = 0; i < 8; ++i) rows[x][s][i / 4][i % 4] = kBack ? f[(at + i) * D + row] : f[row * D + at + i];
            }
    };
    const auto park = [&](uint16_t *to, int x, int ct, f32x4 v) {                       // rows 4g .. of the tile, column 16 ct + c
        const float q[4] = {v[0], v[1], v[2], v[3]};
        const Split3 p = split3(q);
        const int row = 16 * (wave * kEach + x) + 4 * g, at = mat_at<D, true>(16 * ct + c, row / 8) + row % 8;
        *reinterpret_cast<u32x2_t *>(to + at) = p.h;
        *reinterpret_cast<u32x2_t *>(to + kJoin * D + at) = p.m;
        *reinterpret_cast<u32x2_t *>(to + 2 * kJoin * D + at) = p.l;
    };
    constexpr int kColTiles = kJoin / 16;
    f32x4 v[kColTiles][kEach];
    const auto load_tiles = [&](int piece) {                 // what is there of its state; zeros in columns that are none
        const Range r = range_of(state + (size_t)piece * D * a.M, mine ? D : 0, a.M, a.M);
#pragma unroll
        for (int ct = 0; ct < kColTiles; ++ct)
#pragma unroll
            for (int x = 0; x < kEach; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 16 * ct + c < cols ? ((16 * (wave * kEach + x) + 4 * g + i) * a.M + m0 + 16 * ct + c) * 4 : 0x7fffff00;
                    v[ct][x][i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0));
                }
    };
    load_rows(from(0));
    load_tiles(from(0));
    if (mine)
#pragma unroll
        for (int ct = 0; ct < kColTiles; ++ct)
#pragma unroll
            for (int x = 0; x < kEach; ++x) park(sS[0], x, ct, v[ct][x]);
    __syncthreads();
    for (int i = 0; i < count; ++i) {
        const int piece = from(i), to = kBack ? piece - 1 : piece + 1;
        load_tiles(to);
        Parts<3> f[kEach][kSteps];
#pragma unroll
        for (int x = 0; x < kEach; ++x)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) f[x][s] = cut(rows[x][s][0], rows[x][s][1]);
        load_rows(from(i + 1 < count ? i + 1 : i));
        const Range r = range_of(state + (size_t)to * D * a.M, mine ? D : 0, a.M, a.M);
#pragma unroll
        for (int ct = 0; ct < kColTiles; ++ct) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const Parts<3> y = row_operand<D, 3, true>(sS[i & 1], kJoin * D, 16 * ct + c, 4 * s + g);
#pragma unroll
                for (int x = 0; x < kEach; ++x) v[ct][x] = product(f[x][s], y, v[ct][x]);
            }
        }
#pragma unroll
        for (int ct = 0; ct < kColTiles; ++ct)
#pragma unroll
            for (int x = 0; x < kEach; ++x) {
                if (mine) park(sS[(i + 1) & 1], x, ct, v[ct][x]);
                if (16 * ct < cols) store_tile<float>(r, 16 * (wave * kEach + x) + 4 * g, m0 + 16 * ct, a.M, v[ct][x], lane);
            }
        __syncthreads();
    }
}

// ---- one token ------------------------------------------------------------------------------------------
// A workgroup has 64 columns of a head's state, 16 lanes a row (four columns each), 16 rows at a time: the state is read
// once and written once.  k . S and q . S are formed together, o = e^g q . S + (q . k) beta u, so that the sums over the rows meet once.
// Memory bounds it: 512 x 16 heads of 128 x 128 in 209 us, 5.2 TB/s, a copy's rate; 64 x 8 heads of 64 x 64, 17 MB, 4.5 us.
template <typename T, int D> __global__ __launch_bounds__(256) void delta_step_kernel(const DeltaArgs a, float *h) {
    constexpr int kRows = D / 16;
    __shared__ f32x4 red[4][2][16];
    __shared__ alignas(16) float dots[4];
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

void launch_join(const DeltaArgs &a, int dtype, bool back, hipStream_t s) {
    const unsigned grid = (unsigned)(a.B * a.H * ((a.M + kJoin - 1) / kJoin));
    const int C = delta_chunk(dtype);
    float *states = back ? a.piece_dstate : a.piece_state;
#define LA_JOIN(D) back ? delta_join_kernel<D, true><<<grid, 256, 0, s>>>(a, states, C) : delta_join_kernel<D, false><<<grid, 256, 0, s>>>(a, states, C)
    if (a.D == 32) LA_JOIN(32);
    else if (a.D == 64) LA_JOIN(64);
    else LA_JOIN(128);
}

hipError_t launch_delta_fwd(const DeltaArgs &a, int dtype, hipStream_t s) {
    const bool one = a.K == 1 && a.state == nullptr;
    if (one && a.M <= 2 * kCols) {
#define LA_ALL(T, D) delta_fwd_kernel<T, D, kWhole, false, kAll><<<task_grid(a, kWhole), 256, 0, s>>>(a)
        LA_BY_WIDTH(LA_ALL)
        return hipGetLastError();
    }
    const unsigned units = (unsigned)((long)a.B * a.H * a.K);
#define LA_LOCAL(T, D) delta_local_kernel<T, D><<<units, 256, 0, s>>>(a)
    LA_BY_WIDTH(LA_LOCAL)
    if (a.pieces > 1) {
        // where there is a compute unit for each workgroup, LDS that nobody uses keeps two from sharing one (5 x 1531 tokens, 6 heads of
        // 64 x 80 fp32, 240 workgroups: the call 65 us instead of 71)
        const long work = (long)a.B * a.H * ((a.M + kCols - 1) / kCols * (a.pieces - 1) + (a.D + kCols - 1) / kCols * (a.pieces - 2));
        const unsigned grid = task_grid(a, kTransitions), spare = work <= 256 ? 34 * 1024 : 0;
#define LA_PIECES(T, D) delta_fwd_kernel<T, D, kTransitions, false><<<grid, 512, spare, s>>>(a)
        LA_BY_WIDTH(LA_PIECES)
        if (a.pieces > 2) launch_join(a, dtype, false, s);
    }
    if (one) {
#define LA_ALONE(T, D) delta_fwd_kernel<T, D, kWhole, false, kAlone><<<task_grid(a, kWhole), 256, 0, s>>>(a)
        LA_BY_WIDTH(LA_ALONE)
        return hipGetLastError();
    }
#define LA_PASS(T, D) a.state != nullptr ? delta_fwd_kernel<T, D, kWhole, true><<<task_grid(a, kWhole), 512, 0, s>>>(a) : delta_fwd_kernel<T, D, kWhole, false><<<task_grid(a, kWhole), 512, 0, s>>>(a)
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
