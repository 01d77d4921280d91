// Selective state space scan: E channels of S states each,
//   h_t = exp(d_t A) h_{t-1} + d_t x_t B_t,   v_t = C_t . h_t + D x_t,   y_t = v_t z_t sigmoid(z_t),
// with d = softplus(dt + bias) per channel and B_t, C_t [S] shared by the channels of a group; and its gradient
// by the adjoint recurrence
//   g_t = C_t dv_t + exp(d_{t+1} A) g_{t+1},   dx_t = d_t (g_t . B_t) + D dv_t,
//   dd_t = x_t (g_t . B_t) + sum_n A g a h_{t-1},   dA = sum_t d_t g a h_{t-1},   dB_t = sum_e g_t d_t x_t,   dC_t = sum_e dv_t h_t.
//
// A decay per channel and state leaves no matrix product: the work is an exp2 and four vector instructions per
// state and token (12 in the backward, and 4 more to sum dB and dC over lanes), and vector issue is the bound, not memory:
// with the functions, conversions and partial sums of a channel 9 and 25 slots of four cycles a state and token (an exp2
// takes two), which at 8 x 2048 tokens of 2048 channels and 16 states is 121 and 342 us of all SIMDs at 2.4 GHz.  Measured (bf16,
// gated): forward 190 us, the vector units active 65 % of the time, backward 480 us, 77 %; their tensors, 0.40 and
// 0.67 GB with the kept states, take 81 and 135 us at a copy's rate.  So:
// * A lane is a channel, a wave P = 2 (or 4, 8) states of 64 channels, S / P waves a workgroup.  B_t and C_t are then
//   the same in all lanes of a wave: read from LDS at one address for all of them.
// * What a token needs once per channel (softplus, d x, the gate, D x, conversions) is done by all waves together, a
//   tile of 16 tokens at a time, and handed over through LDS; the waves' partial C . h come back the same way.
// * Sequences too few to fill the machine are cut into pieces: the state each piece adds from zero, a scan over the
//   pieces (a piece decays as exp(A sum d)), then the pass itself from the right states.  Twice the exponentials, but the
//   whole machine: one sequence of 32768 x 1024 takes 122 + 7 + 160 us; uncut its 16 workgroups would need 3.0 ms (1.47 us a tile).
#include <type_traits>

#include "la_layer.h"

namespace la {
namespace {

constexpr int T = kScanTile, kLanes = kScanLanes;
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

// Elements of a channel, as they are in memory, for the tokens of a tile that a thread prepares and finishes: wave q takes
// tokens q K .. q K + K - 1 of its 64 channels, so that K tokens of a channel go through LDS side by side.
template <typename TT> struct Raw;
template <> struct Raw<float> { using type = float; };
template <> struct Raw<bf16_t> { using type = uint16_t; };
template <typename TT, int K> struct Column {
    typename Raw<TT>::type v[K];
    // the K tokens from t on of a piece whose first element is *p; tokens behind the last one repeat it.  (No branch: where
    // two ways of loading met, the loads would be waited for.)
    __device__ __forceinline__ void load(const TT *p, unsigned ld, int t, int last) {
        const auto *r = reinterpret_cast<const typename Raw<TT>::type *>(p);
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = r[(uint64_t)(unsigned)min(t + k, last) * ld];
    }
    __device__ __forceinline__ float get(int k) const {
        if constexpr (sizeof(TT) == 2) return __uint_as_float((uint32_t)v[k] << 16);
        else return v[k];
    }
};

// P consecutive states from n0 on of a channel, in the layout of the kept states
template <int P> __device__ __forceinline__ size_t state_at(const ScanArgs &a, int b, int slots, int slot, int n0, int e) {
    return ((((size_t)b * slots + slot) * (a.S / 4) + n0 / 4) * a.E + e) * 4 + n0 % 4;
}

// h of those states, from and to their place p: four side by side, the next four E quads on
template <int P> __device__ __forceinline__ void load_states(float (&h)[P], const float *p, int E) {
    constexpr int V = P < 4 ? P : 4;
#pragma unroll
    for (int n = 0; n < P; n += V) __builtin_memcpy(h + n, p + (size_t)n * E, V * sizeof(float));
}
template <int P> __device__ __forceinline__ void store_states(float *p, const float (&h)[P], int E) {
    constexpr int V = P < 4 ? P : 4;
#pragma unroll
    for (int n = 0; n < P; n += V) __builtin_memcpy(p + (size_t)n * E, h + n, V * sizeof(float));
}

// B_t and C_t of a tile as fp32 pairs in LDS: a wave reads the 2 P values of a token at one address for all its lanes.
// A thread brings kEach values of a tile there, neighbouring threads neighbouring ones.
template <typename TT, int NW, int P> struct Pairs {
    static constexpr int S = NW * P, kEach = 2 * T * S / (64 * NW);        // T * S / 32 / NW: 1, 2 or (four waves of eight states) 4
    float (*lds)[T][S][2];
    const TT *from;                  // this thread's value of the piece's first token
    unsigned ld;
    typename Raw<TT>::type held[2][kEach];
    int t[kEach], which, n;
    // values v = thread + 64 NW i of a tile: token v / (2 S), B before C
    __device__ __forceinline__ Pairs(const ScanArgs &a, const Where &w, float (*l)[T][S][2]) : lds(l) {
        const int c = threadIdx.x % (2 * S);
        which = c / S, n = c % S, ld = which ? a.ldc : a.ldb;
#pragma unroll
        for (int i = 0; i < kEach; ++i) t[i] = (threadIdx.x + 64 * NW * i) / (2 * S);
        from = (const TT *)(which ? a.Ct : a.Bt) + ((size_t)w.b * a.N + w.t0) * ld + (size_t)w.g * S + n;
    }
    __device__ __forceinline__ void fetch(int slot, int i, int last) {     // tile i
        const auto *r = reinterpret_cast<const typename Raw<TT>::type *>(from);
#pragma unroll
        for (int k = 0; k < kEach; ++k) held[slot][k] = r[(uint64_t)(unsigned)min(i * T + t[k], last) * ld];
    }
    __device__ __forceinline__ void park(int slot) const {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if constexpr (sizeof(TT) == 2) lds[slot][t[k]][n][which] = __uint_as_float((uint32_t)held[slot][k] << 16);
            else lds[slot][t[k]][n][which] = held[slot][k];
        }
    }
};
template <int P> struct Pair {
    float v[2 * P];
    __device__ __forceinline__ float B(int n) const { return v[2 * n]; }
    __device__ __forceinline__ float C(int n) const { return v[2 * n + 1]; }
};
template <int P> __device__ __forceinline__ Pair<P> read_pair(const float (*at)[2]) {
    Pair<P> r;
    __builtin_memcpy(r.v, __builtin_assume_aligned(at, 16), sizeof(r.v));
    return r;
}

// kLocal: only what a piece adds to a state of zero, and its sum of d.
// Two buffers in LDS and one barrier a tile: between two barriers a wave finishes tile i - 1 (C . h of all waves, gate,
// store), prepares tile i + 1 and runs tile i, so that one wave's chains of functions hide behind another's states.
// The elements come two tiles ahead (fetched in branches, whose ends wait for all loads: 289 us instead of 190).  B and C by scalar loads, a broadcast
// for free, cost 70 of 265 us in waits for the scalar cache; one state a wave (16 waves) 225 us: more partial sums.
template <typename TT, int NW, int P, bool kLocal> __global__ __launch_bounds__(64 * NW, 2) void scan_fwd_kernel(const ScanArgs a) {
    constexpr int K = T / NW;
    __shared__ __align__(16) float bc[2][T][NW * P][2];
    __shared__ __align__(16) float2 in[2][T / 2][kLanes][2];      // d, d x of two tokens
    __shared__ __align__(16) float out[kLocal ? 1 : 2][kLocal ? 1 : NW][NW][kLanes][K];
    const Where w(a);
    if (kLocal && w.piece == a.pieces - 1) return;                // nothing comes after it
    const int lane = threadIdx.x % 64, q = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n0 = q * P;
    const int e = w.e0 + min(lane, w.channels - 1);               // lanes without a channel repeat the last one's
    const bool live = lane < w.channels;
    float A[P], h[P], sum_d = 0.0f;
#pragma unroll
    for (int n = 0; n < P; ++n) A[n] = a.A[(size_t)e * a.S + n0 + n] * kLog2e, h[n] = 0.0f;
    if constexpr (!kLocal) {
        if (a.pieces > 1) load_states<P>(h, a.piece_h + state_at<P>(a, w.b, a.pieces, w.piece, n0, e), a.E);
        else if (a.h0 != nullptr) __builtin_memcpy(h, a.h0 + ((size_t)w.b * a.E + e) * a.S + n0, sizeof(h));
    }
    const float bias = a.bias == nullptr ? 0.0f : a.bias[e], D = a.D == nullptr ? 0.0f : a.D[e];
    Pairs<TT, NW, P> pairs(a, w, bc);
    const size_t row = (size_t)w.b * a.N + w.t0;
    const bool gated = !kLocal && a.z != nullptr, kept = !kLocal && a.keep != nullptr && live;
    const TT *px = (const TT *)a.x + row * a.ldx + e, *pdt = (const TT *)a.dt + row * a.lddt + e;
    const TT *pz = gated ? (const TT *)a.z + row * a.ldz + e : px;
    const unsigned ldz = gated ? a.ldz : a.ldx;
    TT *py = (TT *)a.y + (row + q * K) * a.E + e;
    float *pk = a.keep + state_at<P>(a, w.b, a.tiles, w.t0 / T, n0, e);
    const int tokens = w.end - w.t0, tiles = tokens > 0 ? (tokens + T - 1) / T : 0;
    // by the tile's parity: elements two tiles ahead, what the store of a tile needs, one tile ahead
    struct Tile { Column<TT, K> x, dt, z; } raw[2];
    struct Ready { float dx[K], gate[K]; } ready[2];
    auto fetch = [&](int slot, int i) {
        const int t = i * T + q * K;
        raw[slot].x.load(px, a.ldx, t, tokens - 1), raw[slot].dt.load(pdt, a.lddt, t, tokens - 1);
        if constexpr (!kLocal) raw[slot].z.load(pz, ldz, t, tokens - 1);
        pairs.fetch(slot, i, tokens - 1);
    };
    auto prepare = [&](int slot, int i) {
        pairs.park(slot);
        const int n = tokens - i * T - q * K;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float x = raw[slot].x.get(k), v = raw[slot].dt.get(k) + bias, sp = softplus(v);
            const float d = k < n ? (a.softplus ? sp : v) : 0.0f; // a step of zero leaves the state as it is
            in[slot][(q * K + k) / 2][lane][(q * K + k) % 2] = make_float2(d, d * x);
            if constexpr (!kLocal) {
                const float z = raw[slot].z.get(k), gate = z * sigmoid(z);
                ready[slot].dx[k] = D * x, ready[slot].gate[k] = gated ? gate : 1.0f;
            }
        }
    };
    auto step = [&](auto parity, int i) {
        constexpr int buf = decltype(parity)::value;
        if (kept) store_states<P>(pk, h, a.E);
        pk += (size_t)a.E * (NW * P);
        fetch(buf, i + 2);                                        // this tile's elements are used up
        float y[T];
#pragma unroll
        for (int j = 0; j < T; ++j) {
            const float2 v = in[buf][j / 2][lane][j % 2];
            const Pair<P> p = read_pair<P>(&bc[buf][j][n0]);
            if constexpr (kLocal) sum_d += v.x;
#pragma unroll
            for (int n = 0; n < P; ++n) {
                h[n] = fmaf(__builtin_amdgcn_exp2f(v.x * A[n]), h[n], v.y * p.B(n));
                y[j] = n == 0 ? p.C(n) * h[n] : fmaf(p.C(n), h[n], y[j]);
            }
            if constexpr (!kLocal) {
                if (j % K == K - 1) __builtin_memcpy(__builtin_assume_aligned(out[buf][q][j / K][lane], 4 * K), &y[j - K + 1], K * sizeof(float));
            }
        }
        prepare(buf ^ 1, i + 1);                                  // behind the last tile: of nothing, read by nobody
        __syncthreads();
        if constexpr (!kLocal) {
            if (a.y == nullptr) return;
            float v[K];
#pragma unroll
            for (int k = 0; k < K; ++k) v[k] = ready[buf].dx[k];
#pragma unroll
            for (int m = 0; m < NW; ++m) {
                float part[K];
                __builtin_memcpy(part, __builtin_assume_aligned(out[buf][m][q][lane], 4 * K), sizeof(part));
#pragma unroll
                for (int k = 0; k < K; ++k) v[k] += part[k];
            }
            const int n = tokens - i * T - q * K, rows = w.t1 - w.t0 - i * T - q * K;
            if (live) {
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    v[k] *= ready[buf].gate[k];
                    if (k < rows) store_elem<false>(py + (size_t)k * a.E, k < n ? v[k] : 0.0f);
                }
            }
            py += (size_t)T * a.E;
        }
    };
    if (tiles > 0) {
        fetch(0, 0);
        fetch(1, 1);
        prepare(0, 0);
    }
    __syncthreads();
    for (int i = 0; i < tiles; i += 2) {
        step(std::integral_constant<int, 0>{}, i);
        if (i + 1 < tiles) step(std::integral_constant<int, 1>{}, i + 1);
    }
    if constexpr (kLocal) {
        if (live) {
            store_states<P>(a.piece_h + state_at<P>(a, w.b, a.pieces, w.piece, n0, e), h, a.E);
            if (q == 0) a.piece_d[((size_t)w.b * a.pieces + w.piece) * a.E + e] = sum_d;
        }
        return;
    }
    if (!live) return;
    if (a.y != nullptr) {                                         // rows behind the sequence
        for (int t = w.t0 + tiles * T + q; t < w.t1; t += NW) store_elem<false>((TT *)a.y + ((size_t)w.b * a.N + t) * a.E + e, 0.0f);
    }
    if (a.h1 != nullptr && w.piece == a.pieces - 1) __builtin_memcpy(a.h1 + ((size_t)w.b * a.E + e) * a.S + n0, h, sizeof(h));
}

// What the pieces add from zero becomes the state before each piece (kReverse: the gradient behind it), in place.  Latency is
// all there is to it (32 pieces of 512 channels and 32 states backwards 6.6 us, 48 of 1024 and 16 forwards 7.5, 0.4 and 0.9 of it for the
// second factor of a decay; 8 ahead and 256 lanes a workgroup took 1.5 and 1.0 more).
template <bool kReverse> __global__ __launch_bounds__(64) void scan_pieces_kernel(const ScanArgs a) {
    constexpr int kAhead = 16;                                    // pieces on their way at a time
    const long per = (long)a.E * a.S;
    for (long id = (long)blockIdx.x * 64 + threadIdx.x; id < a.B * per; id += (long)gridDim.x * 64) {
        const int b = (int)(id / per), e = (int)(id % ((long)a.E * 4) / 4), n = (int)(id % per / ((long)a.E * 4)) * 4 + (int)(id % 4);
        const float A = a.A[(size_t)e * a.S + n] * kLog2e;
        const float *start = kReverse ? a.dh1 : a.h0;
        float h = start == nullptr ? 0.0f : start[((size_t)b * a.E + e) * a.S + n];
        for (int i0 = 0; i0 < a.pieces; i0 += kAhead) {
            float add[kAhead], d[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {                    // behind the last that adds anything: that one once more
                const int at = min(i0 + i, a.pieces - 2), k = kReverse ? a.pieces - 1 - at : at;
                add[i] = a.piece_h[state_at<1>(a, b, a.pieces, k, n, e)];
                d[i] = a.piece_d[((size_t)b * a.pieces + k) * a.E + e];
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (i0 + i >= a.pieces) break;
                const int k = kReverse ? a.pieces - 1 - (i0 + i) : i0 + i;
                a.piece_h[state_at<1>(a, b, a.pieces, k, n, e)] = h;
                // A piece's decay can leave fp32's range where the state behind it does not (growth from a state of zero, which would
                // be inf * 0; a large state that vanishes): so it enters in two factors, of which the second is 1 in between.
                const float power = A * d[i], first = __builtin_amdgcn_fmed3f(power, -126.0f, 126.0f);
                const float rest = __builtin_amdgcn_fmed3f(power - first, -126.0f, 126.0f);
                h = fmaf(__builtin_amdgcn_exp2f(first), __builtin_amdgcn_exp2f(rest) * h, add[i]);
            }
        }
    }
}

// What a piece sends to the piece before it of a gradient of zero behind it: exp(d A) g at its first token, and its sum of d.
template <typename TT, int NW, int P> __global__ __launch_bounds__(64 * NW, 2) void scan_local_bwd_kernel(const ScanArgs a) {
    constexpr int K = T / NW;
    __shared__ __align__(16) float bc[2][T][NW * P][2];
    __shared__ __align__(16) float2 in[2][T / 2][kLanes][2];      // d, dv of two tokens
    const Where w(a);
    if (w.piece == 0) return;                                     // nothing comes before it
    const int lane = threadIdx.x % 64, q = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n0 = q * P;
    const int e = w.e0 + min(lane, w.channels - 1);
    float A[P], g[P], sum_d = 0.0f;
#pragma unroll
    for (int n = 0; n < P; ++n) A[n] = a.A[(size_t)e * a.S + n0 + n] * kLog2e, g[n] = 0.0f;
    const float bias = a.bias == nullptr ? 0.0f : a.bias[e];
    const int tokens = w.end - w.t0, tiles = tokens > 0 ? (tokens + T - 1) / T : 0;
    Pairs<TT, NW, P> pairs(a, w, bc);
    const size_t row = (size_t)w.b * a.N + w.t0;
    const bool gated = a.z != nullptr;
    const TT *pdt = (const TT *)a.dt + row * a.lddt + e, *pdy = (const TT *)a.dy + row * a.E + e;
    const TT *pz = gated ? (const TT *)a.z + row * a.ldz + e : pdt;
    const unsigned ldz = gated ? a.ldz : a.lddt;
    struct Tile { Column<TT, K> dt, dy, z; } raw[2];
    auto fetch = [&](int slot, int i) {                           // before the first tile: the first once more
        const int t = max(i, 0) * T + q * K;
        raw[slot].dt.load(pdt, a.lddt, t, tokens - 1), raw[slot].dy.load(pdy, a.E, t, tokens - 1), raw[slot].z.load(pz, ldz, t, tokens - 1);
        pairs.fetch(slot, max(i, 0), tokens - 1);
    };
    auto prepare = [&](int slot, int i) {
        pairs.park(slot);
        const int n = tokens - i * T - q * K;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float v = raw[slot].dt.get(k) + bias, sp = softplus(v), z = raw[slot].z.get(k), gate = z * sigmoid(z);
            const float d = a.softplus ? sp : v, dv = raw[slot].dy.get(k) * (gated ? gate : 1.0f);
            in[slot][(q * K + k) / 2][lane][(q * K + k) % 2] = make_float2(k < n ? d : 0.0f, k < n ? dv : 0.0f);
        }
    };
    auto step = [&](auto parity, int i) {
        constexpr int buf = decltype(parity)::value;
        fetch(buf, i - 2);
#pragma unroll
        for (int j = T - 1; j >= 0; --j) {
            const float2 v = in[buf][j / 2][lane][j % 2];
            const Pair<P> p = read_pair<P>(&bc[buf][j][n0]);
            sum_d += v.x;
#pragma unroll
            for (int n = 0; n < P; ++n) g[n] = __builtin_amdgcn_exp2f(v.x * A[n]) * fmaf(p.C(n), v.y, g[n]);
        }
        prepare(buf ^ 1, max(i - 1, 0));
        __syncthreads();
    };
    const int first = (tiles - 1) & 1;                            // the last tile's parity
    if (tiles > 0) {
        if (first == 0) fetch(0, tiles - 1), fetch(1, tiles - 2), prepare(0, tiles - 1);
        else fetch(1, tiles - 1), fetch(0, tiles - 2), prepare(1, tiles - 1);
    }
    __syncthreads();
    for (int i = tiles - 1; i >= 0; --i) {
        if (i & 1) {
            step(std::integral_constant<int, 1>{}, i);
            --i;
        }
        step(std::integral_constant<int, 0>{}, i);
    }
    if (lane < w.channels) {
        __builtin_memcpy(a.piece_h + state_at<P>(a, w.b, a.pieces, w.piece, n0, e), g, sizeof(g));
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
// Twice four values over bits 3 and 2 of the lane, v[0 .. 3] to v[0] and v[4 .. 7] to v[1]: a lane gets value 2 bit2 + bit3 of the four,
// summed over the four lanes.  An addition of a moved operand can leave the lanes of some groups of four as they are, and so
// chooses between two values without an instruction of its own: 2 issue slots for each result, where a swap of half a wave
// and the addition take 3, and two selections and a moved addition 3.  So these levels, with the most results, come first (the
// swaps first: 543 us instead of 524 at 8 x 2048 x 2048, 16 states).  What a move reads, here and behind, has to be two slots old:
// hence the order, and the pauses at both ends.  All lanes are active here.
__device__ __forceinline__ void fold_quads(float *v) {
    asm("s_nop 1\n\t"
        "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %0, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %2, %2, %2 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %2, %6, %6 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %3, %3, %3 row_ror:8 row_mask:0xf bank_mask:0x3\n\t"
        "v_add_f32_dpp %3, %7, %7 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
        "v_add_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0x5\n\t"
        "v_add_f32_dpp %0, %1, %1 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
        "v_add_f32_dpp %2, %2, %2 row_half_mirror row_mask:0xf bank_mask:0x5\n\t"
        "v_add_f32_dpp %2, %3, %3 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
        "s_nop 1"
        : "+&v"(v[0]), "+&v"(v[2]), "+&v"(v[4]), "+&v"(v[6])
        : "v"(v[1]), "v"(v[3]), "v"(v[5]), "v"(v[7]));
    v[1] = v[4];
}
// within four lanes; CTRL moves a lane's value to one that differs in the bit (quad permutations)
template <int K, int CTRL> __device__ __forceinline__ void fold_row(float *v, bool bit) {
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const float keep = bit ? v[2 * i + 1] : v[2 * i], send = bit ? v[2 * i] : v[2 * i + 1];
        v[i] = keep + dpp_move<CTRL>(send);
    }
}

// One tile after the other from the last to the first: the states of a tile are formed again from the kept state before
// it and stay in registers (16 tokens x P states, and the decays), then the adjoint runs back over them.  dB and
// dC are sums over channels, which are lanes: the 2 P products of a token are folded over the wave as they appear.
// Between two barriers a wave prepares tile i - 1 and runs tile i; the second barrier only spans the reading of the
// waves' partial sums, whose buffer (98 of the 127 KB) does not fit twice.  Four waves of four states spill; reading the
// partial sums, 10 % of the time, while the next tile is prepared holds more registers (559 us instead of 530 in the same run),
// and the second barrier behind the next tile's states cuts what the compiler overlaps (561 instead of 525).
template <typename TT, int NW, int P> __global__ __launch_bounds__(64 * NW, 2) void scan_bwd_kernel(const ScanArgs a) {
    constexpr int K = T / NW;
    __shared__ __align__(16) float bc[2][T][NW * P][2];
    __shared__ __align__(16) float2 in[2][T / 2][kLanes][2];      // d, d x of two tokens
    __shared__ __align__(16) float in_v[2][T / 2][kLanes][2];     // dv of two tokens
    __shared__ __align__(16) float out[3][NW][NW][kLanes][K];     // g . B, sum A g a h, C . h
    const Where w(a);
    const int lane = threadIdx.x % 64, q = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), n0 = q * P;
    const int e = w.e0 + min(lane, w.channels - 1);               // lanes without a channel repeat the last one's
    const bool live = lane < w.channels;
    float A[P], g[P], dA[P];
#pragma unroll
    for (int n = 0; n < P; ++n) A[n] = a.A[(size_t)e * a.S + n0 + n] * kLog2e, g[n] = dA[n] = 0.0f;
    if (a.pieces > 1) __builtin_memcpy(g, a.piece_h + state_at<P>(a, w.b, a.pieces, w.piece, n0, e), sizeof(g));
    else if (a.dh1 != nullptr) __builtin_memcpy(g, a.dh1 + ((size_t)w.b * a.E + e) * a.S + n0, sizeof(g));
    const float bias = a.bias == nullptr ? 0.0f : a.bias[e], D = a.D == nullptr ? 0.0f : a.D[e];
    float dD = 0.0f, db = 0.0f;
    const int tokens = w.end - w.t0, tiles = tokens > 0 ? (tokens + T - 1) / T : 0, last = w.t0 + (tiles - 1) * T;
    Pairs<TT, NW, P> pairs(a, w, bc);
    const bool gated = a.z != nullptr;
    const size_t row = (size_t)w.b * a.N + w.t0;
    const TT *px = (const TT *)a.x + row * a.ldx + e, *pdt = (const TT *)a.dt + row * a.lddt + e, *pdy = (const TT *)a.dy + row * a.E + e;
    const TT *pz = gated ? (const TT *)a.z + row * a.ldz + e : px;
    const unsigned ldz = gated ? a.ldz : a.ldx;
    size_t dense = (row + (tiles - 1) * T + q * K) * a.E + e;     // of dx, ddt and dz: this thread's first token of a tile
    const float *pk = a.keep + state_at<P>(a, w.b, a.tiles, last / T, n0, e);
    float *pbc = a.part_bc + (((size_t)w.block * a.B + w.b) * a.N + last) * (2 * NW * P) + n0;
    // by the tile's parity: elements two tiles ahead, what the finish of a tile needs, one tile ahead
    struct Tile { Column<TT, K> x, dt, z, dy; } raw[2];
    struct Ready { float d[K], slope[K], x[K], dv[K], dgate[K]; } ready[2];
    float start[2][P] = {};                                       // the kept states before the tiles
    auto fetch = [&](int slot, int i) {                           // before the first tile: the first once more
        const int t = max(i, 0) * T + q * K;
        raw[slot].x.load(px, a.ldx, t, tokens - 1), raw[slot].dt.load(pdt, a.lddt, t, tokens - 1);
        raw[slot].dy.load(pdy, a.E, t, tokens - 1), raw[slot].z.load(pz, ldz, t, tokens - 1);
        pairs.fetch(slot, max(i, 0), tokens - 1);
    };
    auto prepare = [&](int slot, int i) {
        pairs.park(slot);
        __builtin_memcpy(start[slot], pk, sizeof(start[slot]));
        if (i > 0) pk -= (size_t)a.E * (NW * P);
        Ready &r = ready[slot];
        const int n = live ? tokens - i * T - q * K : 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            // behind the sequence and in lanes without a channel: a step of zero, and nothing for any sum
            const bool real = k < n;
            const float raw_d = real ? raw[slot].dt.get(k) + bias : 0.0f, dy = real ? raw[slot].dy.get(k) : 0.0f;
            // softplus and its slope, the sigmoid, from one exponential
            const float ex = __expf(-fabsf(raw_d)), inv = __builtin_amdgcn_rcpf(1.0f + ex), sp = fmaxf(raw_d, 0.0f) + log1p_small(ex);
            const float slope = raw_d >= 0.0f ? inv : ex * inv;
            r.d[k] = real ? (a.softplus ? sp : raw_d) : 0.0f;
            r.slope[k] = a.softplus ? slope : 1.0f;
            r.x[k] = real ? raw[slot].x.get(k) : 0.0f;
            const float z = real ? raw[slot].z.get(k) : 0.0f, gate = sigmoid(z);
            r.dv[k] = dy * (gated ? z * gate : 1.0f);
            r.dgate[k] = dy * gate * fmaf(z, 1.0f - gate, 1.0f);
            const int t = q * K + k;
            in[slot][t / 2][lane][t % 2] = make_float2(r.d[k], r.d[k] * r.x[k]);
            in_v[slot][t / 2][lane][t % 2] = r.dv[k];
        }
    };
    auto step = [&](auto parity, int i) {
        constexpr int buf = decltype(parity)::value;
        float h[T + 1][P], dec[T][P];
#pragma unroll
        for (int n = 0; n < P; ++n) h[0][n] = start[buf][n];
        fetch(buf, i - 2);
#pragma unroll
        for (int j = 0; j < T; ++j) {
            const float2 v = in[buf][j / 2][lane][j % 2];
            const Pair<P> p = read_pair<P>(&bc[buf][j][n0]);
#pragma unroll
            for (int n = 0; n < P; ++n) {
                dec[j][n] = __builtin_amdgcn_exp2f(v.x * A[n]);
                h[j + 1][n] = fmaf(dec[j][n], h[j][n], v.y * p.B(n));
            }
        }
        prepare(buf ^ 1, max(i - 1, 0));
        constexpr int kHeld = P / 2;                              // registers a token's folded products take
        float acc[kHeld * T], sum[3][K], dA_tile[P] = {};         // (a sum of thousands of terms, in two levels)
        float products[8];
#pragma unroll
        for (int j = T - 1; j >= 0; --j) {
            const float2 v = in[buf][j / 2][lane][j % 2];
            const float dv = in_v[buf][j / 2][lane][j % 2];
            const Pair<P> p = read_pair<P>(&bc[buf][j][n0]);
            float gB, gA, y;
            float *prod = P == 2 && j % 2 ? products + 4 : products;
#pragma unroll
            for (int n = 0; n < P; ++n) {
                y = n == 0 ? p.C(n) * h[j + 1][n] : fmaf(p.C(n), h[j + 1][n], y);
                g[n] = fmaf(p.C(n), dv, g[n]);
                gB = n == 0 ? p.B(n) * g[n] : fmaf(p.B(n), g[n], gB);
                prod[n] = g[n] * v.y;
                prod[P + n] = h[j + 1][n] * dv;
                g[n] *= dec[j][n];                                // now the gradient for h_{t-1}
                const float through = g[n] * h[j][n];
                gA = n == 0 ? through * A[n] : fmaf(through, A[n], gA);
                dA_tile[n] = fmaf(through, v.x, dA_tile[n]);
            }
            sum[0][j % K] = gB, sum[1][j % K] = gA, sum[2][j % K] = y;
            if (j % K == 0) {
#pragma unroll
                for (int r = 0; r < 3; ++r) __builtin_memcpy(__builtin_assume_aligned(out[r][q][j / K][lane], 4 * K), sum[r], sizeof(sum[r]));
            }
            if constexpr (P == 4) {
                fold_quads(prod);
                acc[2 * j] = prod[0], acc[2 * j + 1] = prod[1];
            } else if (j % 2 == 0) {                              // with the token before it in this order
                fold_quads(prod);
                acc[j] = prod[0], acc[j + 1] = prod[1];
            }
        }
#pragma unroll
        for (int n = 0; n < P; ++n) dA[n] += dA_tile[n];
        // Lanes that differ in bits 3 and 2 now hold different products: value 4 r + 2 bit2 + bit3 of a token's 2 P.  The
        // other folds choose between the two r (P = 4) by bit 5, and between tokens by the rest.
        fold32<P * T / 4>(acc);
        fold16<P * T / 8>(acc);
        fold_row<P * T / 16, 0x4e>(acc, lane & 2);
        fold_row<P * T / 32, 0xb1>(acc, lane & 1);
#pragma unroll
        for (int k = 0; k < P * T / 32; ++k) {
            const int bit5 = lane >> 5, low = ((lane & 16) >> 4) + (lane & 2) + ((lane & 1) << 2);
            const int j = P == 4 ? k * 8 + low : bit5 + 2 * low;
            const int value = (P == 4 ? 4 * bit5 : 0) + ((lane & 4) >> 1) + ((lane & 8) >> 3);
            if (i * T + j < tokens) pbc[(2 * j + value / P) * (NW * P) + value % P] = acc[k];
        }
        pbc -= T * 2 * NW * P;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 3; ++r) {
#pragma unroll
            for (int k = 0; k < K; ++k) sum[r][k] = 0.0f;
#pragma unroll
            for (int m = 0; m < NW; ++m) {
                float part[K];
                __builtin_memcpy(part, __builtin_assume_aligned(out[r][m][q][lane], 4 * K), sizeof(part));
#pragma unroll
                for (int k = 0; k < K; ++k) sum[r][k] += part[k];
            }
        }
        __syncthreads();
        const Ready &r = ready[buf];
        const int n = live ? tokens - i * T - q * K : 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float gB = sum[0][k], gA = sum[1][k] * (1.0f / kLog2e), y = fmaf(D, r.x[k], sum[2][k]);
            const float ddt = k < n ? fmaf(r.x[k], gB, gA) * r.slope[k] : 0.0f;
            dD = fmaf(r.dv[k], r.x[k], dD), db += ddt;
            if (k < n) {
                const size_t at = dense + (size_t)k * a.E;
                store_elem<false>((TT *)a.dx + at, fmaf(r.d[k], gB, D * r.dv[k]));
                store_elem<false>((TT *)a.ddt + at, ddt);
                if (gated) store_elem<false>((TT *)a.dz + at, r.dgate[k] * y);
            }
        }
        dense -= (size_t)T * a.E;
    };
    const int first = (tiles - 1) & 1;                            // the last tile's parity
    if (tiles > 0) {
        if (first == 0) fetch(0, tiles - 1), fetch(1, tiles - 2), prepare(0, tiles - 1);
        else fetch(1, tiles - 1), fetch(0, tiles - 2), prepare(1, tiles - 1);
    }
    __syncthreads();
    for (int i = tiles - 1; i >= 0; --i) {
        if (i & 1) {
            step(std::integral_constant<int, 1>{}, i);
            --i;
        }
        step(std::integral_constant<int, 0>{}, i);
    }
    if (live) {                                                   // rows behind the sequence
        for (int t = max(w.end, w.t0) + q; t < w.t1; t += NW) {
            const size_t at = ((size_t)w.b * a.N + t) * a.E + e;
            store_elem<false>((TT *)a.dx + at, 0.0f);
            store_elem<false>((TT *)a.ddt + at, 0.0f);
            if (gated) store_elem<false>((TT *)a.dz + at, 0.0f);
        }
    }
    float *sums = a.part + ((size_t)w.b * a.pieces + w.piece) * a.E * (a.S + 2);
    if (live) {
        __builtin_memcpy(sums + (size_t)e * a.S + n0, dA, sizeof(dA));
        if (a.dh0 != nullptr && w.piece == 0) __builtin_memcpy(a.dh0 + ((size_t)w.b * a.E + e) * a.S + n0, g, sizeof(g));
    }
    // dD and the bias's gradient: over the waves, which had different tokens
    float(*red)[NW][kLanes] = reinterpret_cast<float(*)[NW][kLanes]>(&out[0][0][0][0][0]);
    red[0][q][lane] = dD, red[1][q][lane] = db;
    __syncthreads();
    if (q < 2 && live) {
        float v = 0.0f;
#pragma unroll
        for (int m = 0; m < NW; ++m) v += red[q][m][lane];
        sums[(size_t)a.E * (a.S + q) + e] = v;
    }
}

// dB and dC of every token and group: sums over the channel blocks of the group, in their order; zero behind the sequence.
// A thread has 4 of a token's 2 S sums.
template <typename TT> __global__ __launch_bounds__(256) void scan_sum_bc_kernel(const ScanArgs a) {
    constexpr int kAhead = 8;                                     // blocks on their way at a time
    const int per = a.E / a.G, nb = (per + kLanes - 1) / kLanes, quads = a.S / 2;
    const long tokens = (long)a.B * a.N, all = tokens * quads * a.G;
    const size_t block = (size_t)tokens * 2 * a.S;
    for (long id = (long)blockIdx.x * 256 + threadIdx.x; id < all; id += (long)gridDim.x * 256) {
        const long token = id / (quads * a.G);
        const int in_token = (int)(id - token * (quads * a.G)), g = in_token / quads, c = in_token % quads * 4;
        const int b = (int)(token / a.N), t = (int)(token - (long)b * a.N);
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (t < length_of(a.lengths, b, a.N)) {
            const float *from = a.part_bc + (size_t)g * nb * block + (size_t)token * 2 * a.S + c;
            for (int k0 = 0; k0 < nb; k0 += kAhead) {
                f32x4 part[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) part[k] = *reinterpret_cast<const f32x4 *>(from + (size_t)min(k0 + k, nb - 1) * block);
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (k0 + k < nb) v += part[k];
            }
        }
        TT *o = (TT *)(c < a.S ? a.dB : a.dC) + ((size_t)token * a.G + g) * a.S + c % a.S;
        const float f[4] = {v[0], v[1], v[2], v[3]};
        store_row<TT, 4>(o, 4, f);
    }
}

// One token: a lane holds 4 states of a channel, S / 4 neighbouring lanes a channel.  Bound by the states, read and
// written once (512 x 4096 x 16 fp32, 302 MB: 65 us a call, 4.6 TB/s; 49 again on the same states, a part of which the 256 MB
// cache still holds), for few sequences by the launch (64 x 2048: 4 to 6 us).
template <typename TT, int S> __global__ __launch_bounds__(256) void scan_step_kernel(const ScanArgs a, float *__restrict__ h) {
    constexpr int L = S / 4;
    const int wide = (a.E + 256 / L - 1) / (256 / L), b = blockIdx.x / wide;
    const int e = (blockIdx.x - b * wide) * (256 / L) + threadIdx.x / L, q = threadIdx.x % L;
    if (e >= a.E) return;
    const size_t at = (size_t)b * a.E + e, g = (size_t)b * a.G + e / (a.E / a.G);
    float s[4], A[4];
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
// waves of a workgroup and states of a wave
#define LA_SCAN_DISPATCH(S, dtype, ...)                                       \
    do {                                                                      \
        if ((S) == 8) { constexpr int NW = 4, P = 2; LA_SCAN_T(dtype, __VA_ARGS__); }       \
        else if ((S) == 16) { constexpr int NW = 8, P = 2; LA_SCAN_T(dtype, __VA_ARGS__); } \
        else { constexpr int NW = 8, P = 4; LA_SCAN_T(dtype, __VA_ARGS__); }  \
    } while (0)

unsigned blocks_for(long n) { return (unsigned)((n + 255) / 256 < (1 << 20) ? (n + 255) / 256 : 1 << 20); }

}  // namespace

hipError_t launch_scan_fwd(const ScanArgs &a, int dtype, hipStream_t s) {
    const long workgroups = (long)a.B * a.pieces * scan_blocks(a.E, a.G);
    const unsigned grid = (unsigned)workgroups;
    LA_SCAN_DISPATCH(a.S, dtype, {
        if (a.pieces > 1) {
            scan_fwd_kernel<TT, NW, P, true><<<grid, 64 * NW, 0, s>>>(a);
            scan_pieces_kernel<false><<<4 * blocks_for((long)a.B * a.E * a.S), 64, 0, s>>>(a);
        }
        if (NW == 8 && workgroups > scan_cost::kUnits) scan_fwd_kernel<TT, 4, NW * P / 4, false><<<grid, 256, 0, s>>>(a);
        else scan_fwd_kernel<TT, NW, P, false><<<grid, 64 * NW, 0, s>>>(a);
    });
    return hipGetLastError();
}

hipError_t launch_scan_bwd(const ScanArgs &a, int dtype, hipStream_t s) {
    const unsigned grid = (unsigned)((long)a.B * a.pieces * scan_blocks(a.E, a.G));
    LA_SCAN_DISPATCH(a.S, dtype, {
        if (a.pieces > 1) {
            scan_local_bwd_kernel<TT, NW, P><<<grid, 64 * NW, 0, s>>>(a);
            scan_pieces_kernel<true><<<4 * blocks_for((long)a.B * a.E * a.S), 64, 0, s>>>(a);
        }
        scan_bwd_kernel<TT, NW, P><<<grid, 64 * NW, 0, s>>>(a);
    });
    LA_SCAN_T(dtype, scan_sum_bc_kernel<TT><<<blocks_for((long)a.B * a.N * a.G * a.S / 2), 256, 0, s>>>(a));
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
