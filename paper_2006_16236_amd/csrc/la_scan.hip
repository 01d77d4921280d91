// Selective state space scan: E channels of S states each,
//   h_t = exp(d_t A) h_{t-1} + d_t x_t B_t,   v_t = C_t . h_t + D x_t,   y_t = v_t z_t sigmoid(z_t),
// with d = softplus(dt + bias) per channel and B_t, C_t [S] shared by the channels of a group; and its gradient
// by the adjoint recurrence
//   g_t = C_t dv_t + exp(d_{t+1} A) g_{t+1},   dx_t = d_t (g_t . B_t) + D dv_t,
//   dd_t = x_t (g_t . B_t) + sum_n A g a h_{t-1},   dA = sum_t d_t g a h_{t-1},   dB_t = sum_e g_t d_t x_t,   dC_t = sum_e dv_t h_t.
//
// A decay per channel and state leaves no matrix product: the work is an exp2 and four vector instructions per
// state and token (13 in the backward), and vector issue is the bound, not memory.  So:
// * A lane is a channel, a wave kScanPer = 4 states of 64 channels, S / 4 waves a workgroup.  B_t and C_t are then the
//   same in all lanes of a wave: they come through the scalar unit and enter the vector instructions as
//   scalar operands, with no vector load, LDS read or register of their own.
// * What a token needs once per channel (softplus, d x, the gate, D x, conversions) is done by all waves together, a
//   tile of 16 tokens at a time, and handed over through LDS; the waves' partial C . h come back the same way.
// * Sequences too few to fill the machine are cut into pieces: the state each piece adds from zero, a scan over the
//   pieces (a piece decays as exp(A sum d)), then the pass itself from the right states.
#include "la_layer.h"

namespace la {
namespace {

constexpr int T = kScanTile, kLanes = kScanLanes, P = kScanPer;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ int length_of(const int *lengths, int b, int N) {
    return lengths == nullptr ? N : min(max(lengths[b], 0), N);
}

// Which part of the problem a workgroup has: 64 channels of a group, one sequence, one piece of it.
struct Where {
    int b, g, e0, channels, piece, block, len, t0, t1, end;       // tokens [t0, t1) of the piece, [t0, end) of the sequence
    __device__ __forceinline__ Where(const ScanArgs &a) {
        const int per = a.E / a.G, nb = (per + kLanes - 1) / kLanes;
        long id = blockIdx.x;
        block = (int)(id % (nb * a.G)), id /= nb * a.G;
        piece = (int)(id % a.pieces), b = (int)(id / a.pieces);
        g = block / nb;
        const int c0 = (block % nb) * kLanes;
        e0 = g * per + c0, channels = min(kLanes, per - c0);
        len = length_of(a.lengths, b, a.N);
        t0 = piece * a.piece_tiles * T, t1 = min(a.N, t0 + a.piece_tiles * T), end = min(t1, len);
    }
};

// The elements of a tile that a thread prepares and finishes: EPT channels of one token.
template <typename TT, int NW> struct Mine {
    static constexpr int EPT = T * kLanes / (64 * NW);            // 8, 4, 2 for 2, 4, 8 waves
    int t, c, valid;
    __device__ __forceinline__ Mine(int channels) {
        t = threadIdx.x / (kLanes / EPT), c = threadIdx.x % (kLanes / EPT) * EPT, valid = channels - c;
    }
};

__device__ __forceinline__ size_t state_at(const ScanArgs &a, int b, int slots, int slot, int q, int e) {
    return ((((size_t)b * slots + slot) * (a.S / P) + q) * a.E + e) * P;
}

// B_t or C_t of a wave's states
template <typename TT> using Row = Words<P * sizeof(TT) / 4>;
template <typename TT> __device__ __forceinline__ Row<TT> row_of(const void *base, long ld, size_t first, int t, int last) {
    return load_uniform<P * sizeof(TT) / 4>(base, (first + (size_t)min(t, last) * ld) * sizeof(TT));
}

// kLocal: only what a piece adds to a state of zero, and its sum of d
template <typename TT, int NW, bool kLocal> __global__ __launch_bounds__(64 * NW) void scan_fwd_kernel(const ScanArgs a) {
    using M = Mine<TT, NW>;
    constexpr int EPT = M::EPT;
    __shared__ float2 in[T][kLanes];                              // d, d x
    __shared__ float out[kLocal ? 1 : NW][T][kLanes];
    const Where w(a);
    const M me(w.channels);
    if (kLocal && w.piece == a.pieces - 1) return;                // nothing comes after it
    const int lane = threadIdx.x % 64, q = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int e = w.e0 + min(lane, w.channels - 1);               // lanes without a channel repeat the last one's
    const bool live = lane < w.channels;
    float A[P], h[P], sum_d = 0.0f;
#pragma unroll
    for (int n = 0; n < P; ++n) A[n] = a.A[(size_t)e * a.S + q * P + n] * kLog2e, h[n] = 0.0f;
    if constexpr (!kLocal) {
        if (a.pieces > 1) __builtin_memcpy(h, a.piece_h + state_at(a, w.b, a.pieces, w.piece, q, e), sizeof(h));
        else if (a.h0 != nullptr) __builtin_memcpy(h, a.h0 + ((size_t)w.b * a.E + e) * a.S + q * P, sizeof(h));
    }
    float bias[EPT], D[EPT];
    load_params<EPT>(a.bias == nullptr ? nullptr : a.bias + w.e0 + me.c, me.valid, bias);
    load_params<EPT>(a.D == nullptr ? nullptr : a.D + w.e0 + me.c, me.valid, D);
    const size_t row0 = (size_t)w.b * a.N;
    const size_t bfirst = row0 * a.ldb + (size_t)w.g * a.S + q * P, cfirst = row0 * a.ldc + (size_t)w.g * a.S + q * P;

    Piece<TT, EPT> x, dt, z{};
    auto fetch = [&](int t) {
        const size_t r = row0 + t + me.t;
        const int valid = t + me.t < w.end ? me.valid : 0;
        x = load_piece<TT, EPT>((const TT *)a.x + r * a.ldx + w.e0 + me.c, valid);
        dt = load_piece<TT, EPT>((const TT *)a.dt + r * a.lddt + w.e0 + me.c, valid);
        if (!kLocal && a.z != nullptr) z = load_piece<TT, EPT>((const TT *)a.z + r * a.ldz + w.e0 + me.c, valid);
    };
    fetch(w.t0);
    for (int t = w.t0; t < w.end; t += T) {
        const Piece<TT, EPT> xt = x, zt = z;
        const bool real = t + me.t < w.end;
#pragma unroll
        for (int i = 0; i < EPT; ++i) {
            float d = dt.get(i) + bias[i];
            if (a.softplus) d = softplus(d);
            if (!real) d = 0.0f;                                  // a step of zero leaves the state as it is
            in[me.t][me.c + i] = make_float2(d, d * x.get(i));
        }
        __syncthreads();
        if (t + T < w.end) fetch(t + T);
        if (!kLocal && a.keep != nullptr && live)
            __builtin_memcpy(a.keep + state_at(a, w.b, a.tiles, t / T, q, e), h, sizeof(h));
#pragma unroll
        for (int j = 0; j < T; ++j) {
            const float2 v = in[j][lane];
            const Row<TT> B = row_of<TT>(a.Bt, a.ldb, bfirst, t + j, w.end - 1);
            float y = 0.0f;
            if constexpr (kLocal) {
                sum_d += v.x;
#pragma unroll
                for (int n = 0; n < P; ++n) h[n] = fmaf(__builtin_amdgcn_exp2f(v.x * A[n]), h[n], v.y * word_value<TT, P>(B, n));
            } else {
                const Row<TT> C = row_of<TT>(a.Ct, a.ldc, cfirst, t + j, w.end - 1);
#pragma unroll
                for (int n = 0; n < P; ++n) {
                    h[n] = fmaf(__builtin_amdgcn_exp2f(v.x * A[n]), h[n], v.y * word_value<TT, P>(B, n));
                    y = fmaf(word_value<TT, P>(C, n), h[n], y);
                }
                out[q][j][lane] = y;
            }
        }
        __syncthreads();
        if constexpr (!kLocal) {
            if (a.y != nullptr && t + me.t < w.t1) {
                float o[EPT];
#pragma unroll
                for (int i = 0; i < EPT; ++i) {
                    float v = D[i] * xt.get(i);
#pragma unroll
                    for (int k = 0; k < NW; ++k) v += out[k][me.t][me.c + i];
                    if (a.z != nullptr) v *= zt.get(i) * sigmoid(zt.get(i));
                    o[i] = real ? v : 0.0f;
                }
                store_row<TT, EPT>((TT *)a.y + (row0 + t + me.t) * a.E + w.e0 + me.c, me.valid, o);
            }
        }
    }
    if constexpr (kLocal) {
        if (live) {
            __builtin_memcpy(a.piece_h + state_at(a, w.b, a.pieces, w.piece, q, e), h, sizeof(h));
            if (q == 0) a.piece_d[((size_t)w.b * a.pieces + w.piece) * a.E + e] = sum_d;
        }
        return;
    }
    if (a.y != nullptr) {                                         // rows behind the sequence
        const float zero[EPT] = {};
        const int done = w.end > w.t0 ? w.t0 + (w.end - w.t0 + T - 1) / T * T : w.t0;
        for (int t = done + me.t; t < w.t1; t += T) store_row<TT, EPT>((TT *)a.y + (row0 + t) * a.E + w.e0 + me.c, me.valid, zero);
    }
    if (a.h1 != nullptr && w.piece == a.pieces - 1 && live)
        __builtin_memcpy(a.h1 + ((size_t)w.b * a.E + e) * a.S + q * P, h, sizeof(h));
}

// What the pieces add from zero becomes the state before each piece (kReverse: the gradient behind it), in place.
template <bool kReverse> __global__ __launch_bounds__(256) void scan_pieces_kernel(const ScanArgs a) {
    const long per = (long)a.E * a.S;
    for (long id = (long)blockIdx.x * 256 + threadIdx.x; id < a.B * per; id += (long)gridDim.x * 256) {
    const int b = (int)(id / per), q = (int)(id % per / ((long)a.E * P)), e = (int)(id % ((long)a.E * P) / P), n = (int)(id % P);
    const float A = a.A[(size_t)e * a.S + q * P + n] * kLog2e;
    const float *start = kReverse ? a.dh1 : a.h0;
    float h = start == nullptr ? 0.0f : start[((size_t)b * a.E + e) * a.S + q * P + n];
    for (int i = 0; i < a.pieces; ++i) {
        const int k = kReverse ? a.pieces - 1 - i : i;
        float *at = a.piece_h + state_at(a, b, a.pieces, k, q, e) + n;
        if (i + 1 == a.pieces) {                                  // nothing is added behind the last
            *at = h;
            break;
        }
        const float add = *at;
        *at = h;
        h = fmaf(__builtin_amdgcn_exp2f(A * a.piece_d[((size_t)b * a.pieces + k) * a.E + e]), h, add);
    }
    }
}

// What a piece sends to the piece before it of a gradient of zero behind it: exp(d A) g at its first token, and its sum of d.
template <typename TT, int NW> __global__ __launch_bounds__(64 * NW) void scan_local_bwd_kernel(const ScanArgs a) {
    using M = Mine<TT, NW>;
    constexpr int EPT = M::EPT;
    __shared__ float2 in[T][kLanes];                              // d, dv
    const Where w(a);
    if (w.piece == 0) return;                                     // nothing comes before it
    const M me(w.channels);
    const int lane = threadIdx.x % 64, q = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int e = w.e0 + min(lane, w.channels - 1);
    float A[P], g[P], sum_d = 0.0f;
#pragma unroll
    for (int n = 0; n < P; ++n) A[n] = a.A[(size_t)e * a.S + q * P + n] * kLog2e, g[n] = 0.0f;
    float bias[EPT];
    load_params<EPT>(a.bias == nullptr ? nullptr : a.bias + w.e0 + me.c, me.valid, bias);
    const size_t row0 = (size_t)w.b * a.N, cfirst = row0 * a.ldc + (size_t)w.g * a.S + q * P;
    const int tiles = w.end > w.t0 ? (w.end - w.t0 + T - 1) / T : 0;
    for (int i = tiles - 1; i >= 0; --i) {
        const int t = w.t0 + i * T;
        const size_t r = row0 + t + me.t;
        const int valid = t + me.t < w.end ? me.valid : 0;
        const Piece<TT, EPT> dt = load_piece<TT, EPT>((const TT *)a.dt + r * a.lddt + w.e0 + me.c, valid);
        const Piece<TT, EPT> dy = load_piece<TT, EPT>((const TT *)a.dy + r * a.E + w.e0 + me.c, valid);
        Piece<TT, EPT> z{};
        if (a.z != nullptr) z = load_piece<TT, EPT>((const TT *)a.z + r * a.ldz + w.e0 + me.c, valid);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < EPT; ++k) {
            float d = dt.get(k) + bias[k], dv = dy.get(k);
            if (a.softplus) d = softplus(d);
            if (a.z != nullptr) dv *= z.get(k) * sigmoid(z.get(k));
            in[me.t][me.c + k] = make_float2(t + me.t < w.end ? d : 0.0f, t + me.t < w.end ? dv : 0.0f);
        }
        __syncthreads();
#pragma unroll
        for (int j = T - 1; j >= 0; --j) {
            const float2 v = in[j][lane];
            const Row<TT> C = row_of<TT>(a.Ct, a.ldc, cfirst, t + j, w.end - 1);
            sum_d += v.x;
#pragma unroll
            for (int n = 0; n < P; ++n) g[n] = __builtin_amdgcn_exp2f(v.x * A[n]) * fmaf(word_value<TT, P>(C, n), v.y, g[n]);
        }
    }
    if (lane < w.channels) {
        __builtin_memcpy(a.piece_h + state_at(a, w.b, a.pieces, w.piece, q, e), g, sizeof(g));
        if (q == 0) a.piece_d[((size_t)w.b * a.pieces + w.piece) * a.E + e] = sum_d;
    }
}

// Sums of 2 K values over 64 lanes, halving the number of values with every step: lanes with the bit keep the second
// of a pair, the others the first.  v[2i], v[2i + 1] -> v[i]
template <int K> __device__ __forceinline__ void fold32(float *v) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const u32x2_pair r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}
template <int K> __device__ __forceinline__ void fold16(float *v) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const u32x2_pair r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}
// within 16 lanes; CTRL moves a lane's value to one that differs in the bit (row_ror 8, half mirror, quad permutations)
template <int K, int CTRL> __device__ __forceinline__ void fold_row(float *v, bool bit) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const float keep = bit ? v[2 * i + 1] : v[2 * i], send = bit ? v[2 * i] : v[2 * i + 1];
        v[i] = keep + dpp_move<CTRL>(send);
    }
}

// One tile after the other from the last to the first: the states of a tile are formed again from the kept state before
// it and stay in registers (16 tokens x 4 states, and the decays), then the adjoint runs back over them.  dB and
// dC are sums over channels, which are lanes: the 8 products of a token are folded over the wave as they appear.
template <typename TT, int NW> __global__ __launch_bounds__(64 * NW, 2) void scan_bwd_kernel(const ScanArgs a) {
    using M = Mine<TT, NW>;
    constexpr int EPT = M::EPT;
    __shared__ float2 in[T][kLanes];                              // d, d x
    __shared__ float in_v[T][kLanes];                             // dv
    __shared__ float out[3][NW][T][kLanes];                       // g . B, sum A g a h, C . h
    const Where w(a);
    const M me(w.channels);
    const int lane = threadIdx.x % 64, q = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int e = w.e0 + min(lane, w.channels - 1);
    const bool live = lane < w.channels;
    float A[P], g[P], dA[P];
#pragma unroll
    for (int n = 0; n < P; ++n) A[n] = a.A[(size_t)e * a.S + q * P + n] * kLog2e, g[n] = dA[n] = 0.0f;
    if (a.pieces > 1) __builtin_memcpy(g, a.piece_h + state_at(a, w.b, a.pieces, w.piece, q, e), sizeof(g));
    else if (a.dh1 != nullptr) __builtin_memcpy(g, a.dh1 + ((size_t)w.b * a.E + e) * a.S + q * P, sizeof(g));
    float bias[EPT], D[EPT], dD[EPT] = {}, db[EPT] = {};
    load_params<EPT>(a.bias == nullptr ? nullptr : a.bias + w.e0 + me.c, me.valid, bias);
    load_params<EPT>(a.D == nullptr ? nullptr : a.D + w.e0 + me.c, me.valid, D);
    const size_t row0 = (size_t)w.b * a.N;
    const size_t bfirst = row0 * a.ldb + (size_t)w.g * a.S + q * P, cfirst = row0 * a.ldc + (size_t)w.g * a.S + q * P;
    const int tiles = w.end > w.t0 ? (w.end - w.t0 + T - 1) / T : 0;
    const bool gated = a.z != nullptr;

    Piece<TT, EPT> x, dt, z{}, dy;
    auto fetch = [&](int t) {
        const size_t r = row0 + t + me.t;
        const int valid = t + me.t < w.end ? me.valid : 0;
        x = load_piece<TT, EPT>((const TT *)a.x + r * a.ldx + w.e0 + me.c, valid);
        dt = load_piece<TT, EPT>((const TT *)a.dt + r * a.lddt + w.e0 + me.c, valid);
        dy = load_piece<TT, EPT>((const TT *)a.dy + r * a.E + w.e0 + me.c, valid);
        if (gated) z = load_piece<TT, EPT>((const TT *)a.z + r * a.ldz + w.e0 + me.c, valid);
    };
    if (tiles > 0) fetch(w.t0 + (tiles - 1) * T);
    for (int i = tiles - 1; i >= 0; --i) {
        const int t = w.t0 + i * T;
        const bool real = t + me.t < w.end;
        const Piece<TT, EPT> xt = x, zt = z, dyt = dy;
        float d[EPT], slope[EPT], gate[EPT];
#pragma unroll
        for (int k = 0; k < EPT; ++k) {
            const float raw = dt.get(k) + bias[k];
            d[k] = real ? (a.softplus ? softplus(raw) : raw) : 0.0f;
            slope[k] = real ? (a.softplus ? sigmoid(raw) : 1.0f) : 0.0f;
            gate[k] = sigmoid(zt.get(k));
            const float dv = gated ? dyt.get(k) * zt.get(k) * gate[k] : dyt.get(k);
            in[me.t][me.c + k] = make_float2(d[k], d[k] * xt.get(k));
            in_v[me.t][me.c + k] = real ? dv : 0.0f;
        }
        __syncthreads();
        float h[T + 1][P], dec[T][P];
        __builtin_memcpy(h[0], a.keep + state_at(a, w.b, a.tiles, t / T, q, e), sizeof(h[0]));
        if (i > 0) fetch(t - T);
#pragma unroll
        for (int j = 0; j < T; ++j) {
            const float2 v = in[j][lane];
            const Row<TT> B = row_of<TT>(a.Bt, a.ldb, bfirst, t + j, w.end - 1);
#pragma unroll
            for (int n = 0; n < P; ++n) {
                dec[j][n] = __builtin_amdgcn_exp2f(v.x * A[n]);
                h[j + 1][n] = fmaf(dec[j][n], h[j][n], v.y * word_value<TT, P>(B, n));
            }
        }
        float acc[2 * T];                                         // two registers a token, each a value per 16 lanes
#pragma unroll
        for (int j = T - 1; j >= 0; --j) {
            const float2 v = in[j][lane];
            const float dv = in_v[j][lane];
            const Row<TT> B = row_of<TT>(a.Bt, a.ldb, bfirst, t + j, w.end - 1);
            const Row<TT> C = row_of<TT>(a.Ct, a.ldc, cfirst, t + j, w.end - 1);
            float gB = 0.0f, gA = 0.0f, y = 0.0f, bc[2 * P];
#pragma unroll
            for (int n = 0; n < P; ++n) {
                y = fmaf(word_value<TT, P>(C, n), h[j + 1][n], y);
                g[n] = fmaf(word_value<TT, P>(C, n), dv, g[n]);
                gB = fmaf(word_value<TT, P>(B, n), g[n], gB);
                bc[n] = live ? g[n] * v.y : 0.0f;
                bc[P + n] = live ? h[j + 1][n] * dv : 0.0f;
                g[n] *= dec[j][n];                                // now the gradient for h_{t-1}
                const float through = g[n] * h[j][n];
                gA = fmaf(through, A[n], gA);
                dA[n] = fmaf(through, v.x, dA[n]);
            }
            out[0][q][j][lane] = gB;
            out[1][q][j][lane] = gA;
            if (gated) out[2][q][j][lane] = y;
            fold32<P>(bc);
            fold16<P / 2>(bc);
            acc[2 * j] = bc[0], acc[2 * j + 1] = bc[1];
        }
        fold_row<T, 0x128>(acc, lane & 8);
        fold_row<T / 2, 0x141>(acc, lane & 4);
        fold_row<T / 4, 0x4e>(acc, lane & 2);
        fold_row<T / 8, 0xb1>(acc, lane & 1);
        // Which value a lane ends up with: register pair (2j, 2j + 1) held, by bits 5 and 4 of the lane, values
        // {bc[4r + 2 bit4 + bit5]}; the folds chose r by bit 3 and the token by bits 2, 1, 0 of the lane and the register.
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int j = k * 8 + ((lane & 1) << 2) + (lane & 2) + ((lane & 4) >> 2);
            const int value = ((lane & 8) >> 1) + ((lane & 16) >> 3) + ((lane & 32) >> 5);
            if (t + j < w.end) {
                const int which = value / P, n = q * P + value % P;
                a.part_bc[((((size_t)w.block * a.B + w.b) * a.N + t + j) * 2 + which) * a.S + n] = acc[k];
            }
        }
        __syncthreads();
        if (real) {
            float o[EPT], od[EPT], oz[EPT];
#pragma unroll
            for (int k = 0; k < EPT; ++k) {
                float gB = 0.0f, gA = 0.0f, y = 0.0f;
#pragma unroll
                for (int m = 0; m < NW; ++m) {
                    gB += out[0][m][me.t][me.c + k];
                    gA += out[1][m][me.t][me.c + k];
                    if (gated) y += out[2][m][me.t][me.c + k];
                }
                const float xv = xt.get(k), zv = zt.get(k), dyv = dyt.get(k), dv = gated ? dyv * zv * gate[k] : dyv;
                o[k] = fmaf(d[k], gB, D[k] * dv);
                od[k] = fmaf(xv, gB, gA * (1.0f / kLog2e)) * slope[k];
                y = fmaf(D[k], xv, y);
                oz[k] = dyv * y * gate[k] * fmaf(zv, 1.0f - gate[k], 1.0f);
                dD[k] = fmaf(dv, xv, dD[k]);
                db[k] += od[k];
            }
            const size_t at = (row0 + t + me.t) * a.E + w.e0 + me.c;
            store_row<TT, EPT>((TT *)a.dx + at, me.valid, o);
            store_row<TT, EPT>((TT *)a.ddt + at, me.valid, od);
            if (gated) store_row<TT, EPT>((TT *)a.dz + at, me.valid, oz);
        }
    }
    {   // rows behind the sequence
        const float zero[EPT] = {};
        for (int t = max(w.end, w.t0) + me.t; t < w.t1; t += T) {
            const size_t at = (row0 + t) * a.E + w.e0 + me.c;
            store_row<TT, EPT>((TT *)a.dx + at, me.valid, zero);
            store_row<TT, EPT>((TT *)a.ddt + at, me.valid, zero);
            if (gated) store_row<TT, EPT>((TT *)a.dz + at, me.valid, zero);
        }
    }
    float *sums = a.part + ((size_t)w.b * a.pieces + w.piece) * a.E * (a.S + 2);
    if (live) {
        __builtin_memcpy(sums + (size_t)e * a.S + q * P, dA, sizeof(dA));
        if (a.dh0 != nullptr && w.piece == 0) __builtin_memcpy(a.dh0 + ((size_t)w.b * a.E + e) * a.S + q * P, g, sizeof(g));
    }
    // dD and the bias's gradient: over the 16 tokens of the tile's rows
    float *red = &out[0][0][0][0];                                // [2][T][64]
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EPT; ++k) red[me.t * kLanes + me.c + k] = dD[k], red[(T + me.t) * kLanes + me.c + k] = db[k];
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * kLanes; c += 64 * NW) {
        const int ch = c % kLanes, which = c / kLanes;
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < T; ++j) v += red[(which * T + j) * kLanes + ch];
        if (ch < w.channels) sums[(size_t)a.E * (a.S + which) + w.e0 + ch] = v;
    }
}

// dB and dC of every token and group: sums over the channel blocks of the group; zero behind the sequence
template <typename TT> __global__ __launch_bounds__(256) void scan_sum_bc_kernel(const ScanArgs a) {
    const int per = a.E / a.G, nb = (per + kLanes - 1) / kLanes;
    const long row = (long)a.B * a.N, all = row * 2 * a.S * a.G;
    for (long id = (long)blockIdx.x * 256 + threadIdx.x; id < all; id += (long)gridDim.x * 256) {
        const long rows = id / (2 * a.S * a.G);
        const int in_row = (int)(id - rows * (2 * a.S * a.G)), g = in_row / (2 * a.S), c = in_row % (2 * a.S);
        const int b = (int)(rows / a.N), t = (int)(rows - (long)b * a.N);
        float v = 0.0f;
        if (t < length_of(a.lengths, b, a.N))
            for (int k = 0; k < nb; ++k) v += a.part_bc[(((size_t)(g * nb + k)) * row + rows) * 2 * a.S + c];
        TT *o = (TT *)(c < a.S ? a.dB : a.dC);
        store_elem<false>(o + ((size_t)rows * a.G + g) * a.S + c % a.S, v);
    }
}

// One token: a lane holds 4 states of a channel, S / 4 neighbouring lanes a channel.  Bound by the states, read and
// written once.
template <typename TT, int S> __global__ __launch_bounds__(256) void scan_step_kernel(const ScanArgs a, float *__restrict__ h) {
    constexpr int L = S / 4;
    const int wide = (a.E + 256 / L - 1) / (256 / L), b = blockIdx.x / wide;
    const int e = (blockIdx.x - b * wide) * (256 / L) + threadIdx.x / L, q = threadIdx.x % L;
    if (e >= a.E) return;
    const size_t at = (size_t)b * a.E + e, g = (size_t)b * a.G + e / (a.E / a.G);
    float s[4], A[4], B[4], C[4];
    __builtin_memcpy(s, h + at * S + q * 4, sizeof(s));
    __builtin_memcpy(A, a.A + (size_t)e * S + q * 4, sizeof(A));
    const Piece<TT, 4> pb = load_piece<TT, 4>((const TT *)a.Bt + g * S + q * 4, 4), pc = load_piece<TT, 4>((const TT *)a.Ct + g * S + q * 4, 4);
    const float x = to_f32(((const TT *)a.x)[at]);
    float d = to_f32(((const TT *)a.dt)[at]) + (a.bias != nullptr ? a.bias[e] : 0.0f);
    if (a.softplus) d = softplus(d);
    float y = 0.0f;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        s[n] = fmaf(__builtin_amdgcn_exp2f(d * (A[n] * kLog2e)), s[n], d * x * pb.get(n));
        y = fmaf(pc.get(n), s[n], y);
    }
    __builtin_memcpy(h + at * S + q * 4, s, sizeof(s));
    if constexpr (L >= 2) y += dpp_move<0xb1>(y);
    if constexpr (L >= 4) y += dpp_move<0x4e>(y);
    if constexpr (L >= 8) y += dpp_move<0x141>(y);
    if (q == 0) {
        if (a.D != nullptr) y = fmaf(a.D[e], x, y);
        if (a.z != nullptr) {
            const float z = to_f32(((const TT *)a.z)[at]);
            y *= z * sigmoid(z);
        }
        store_elem<false>((TT *)a.y + at, y);
    }
}

#define LA_SCAN_T(dtype, ...)                                                 \
    do {                                                                      \
        if ((dtype) == 0) { using TT = float; __VA_ARGS__; }                  \
        else { using TT = bf16_t; __VA_ARGS__; }                              \
    } while (0)
#define LA_SCAN_DISPATCH(S, dtype, ...)                                       \
    do {                                                                      \
        if ((S) == 8) { constexpr int NW = 2; LA_SCAN_T(dtype, __VA_ARGS__); }       \
        else if ((S) == 16) { constexpr int NW = 4; LA_SCAN_T(dtype, __VA_ARGS__); } \
        else { constexpr int NW = 8; LA_SCAN_T(dtype, __VA_ARGS__); }         \
    } while (0)

unsigned blocks_for(long n) { return (unsigned)((n + 255) / 256 < (1 << 20) ? (n + 255) / 256 : 1 << 20); }

}  // namespace

int scan_blocks(int E, int G) { return G * ((E / G + kLanes - 1) / kLanes); }

void scan_cut(ScanArgs &a) {
    a.tiles = (a.N + T - 1) / T;
    const long whole = (long)a.B * scan_blocks(a.E, a.G);
    long pieces = 1;
    if (whole < 160) pieces = (512 + whole - 1) / whole;
    const long most = a.tiles / 4 > 1 ? a.tiles / 4 : 1;          // no piece shorter than 64 tokens
    if (pieces > most) pieces = most;
    a.piece_tiles = (int)((a.tiles + pieces - 1) / pieces);
    a.pieces = (a.tiles + a.piece_tiles - 1) / a.piece_tiles;
}

hipError_t launch_scan_fwd(const ScanArgs &a, int dtype, hipStream_t s) {
    const unsigned grid = (unsigned)((long)a.B * a.pieces * scan_blocks(a.E, a.G));
    LA_SCAN_DISPATCH(a.S, dtype, {
        if (a.pieces > 1) {
            scan_fwd_kernel<TT, NW, true><<<grid, 64 * NW, 0, s>>>(a);
            scan_pieces_kernel<false><<<blocks_for((long)a.B * a.E * a.S), 256, 0, s>>>(a);
        }
        scan_fwd_kernel<TT, NW, false><<<grid, 64 * NW, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_scan_bwd(const ScanArgs &a, int dtype, hipStream_t s) {
    const unsigned grid = (unsigned)((long)a.B * a.pieces * scan_blocks(a.E, a.G));
    LA_SCAN_DISPATCH(a.S, dtype, {
        if (a.pieces > 1) {
            scan_local_bwd_kernel<TT, NW><<<grid, 64 * NW, 0, s>>>(a);
            scan_pieces_kernel<true><<<blocks_for((long)a.B * a.E * a.S), 256, 0, s>>>(a);
        }
        scan_bwd_kernel<TT, NW><<<grid, 64 * NW, 0, s>>>(a);
        scan_sum_bc_kernel<TT><<<blocks_for((long)a.B * a.N * a.G * 2 * a.S), 256, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_scan_step(const ScanArgs &a, float *h, int dtype, hipStream_t s) {
    const int per = 256 / (a.S / 4);
    const unsigned grid = (unsigned)((long)((a.E + per - 1) / per) * a.B);
    LA_SCAN_T(dtype, {
        if (a.S == 8) scan_step_kernel<TT, 8><<<grid, 256, 0, s>>>(a, h);
        else if (a.S == 16) scan_step_kernel<TT, 16><<<grid, 256, 0, s>>>(a, h);
        else scan_step_kernel<TT, 32><<<grid, 256, 0, s>>>(a, h);
    });
    return hipGetLastError();
}

}  // namespace la
