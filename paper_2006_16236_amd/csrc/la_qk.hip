// Norm of queries and keys for each head and the position rotation, in one pass (la_qk_*).
//
// A head of D = 8 G' elements is held by G lanes (G' rounded up to a power of two), eight elements each, so that both
// elements of a pair that is turned together sit in one lane: a lane has four elements of the first half of the turned
// part and the four that go with them of the second, or eight neighbours.  Sums over a head are sums over G lanes.
// A wave takes the heads of one token 64 / G at a time: its lanes' four angles are then formed once per token, and the
// queries and keys of a token are one list of H + Hk heads.
// Memory bounds both directions: 8 x 2048 tokens, 16 + 16 heads of 128 bf16, forward 50 us (5.3 TB/s), backward 85 (4.7 TB/s); one
// token of 64 sequences, 8 + 8 heads of 64, is 4.5 us, the launch and two trips to memory.
#include <hip/hip_runtime.h>

#include "la_mixer.h"

namespace la {
namespace {

// Four elements as they are in memory, at any address.
template <typename T> struct Quad {
    uint32_t w[sizeof(T)];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};
template <typename T> __device__ __forceinline__ Quad<T> load_quad(const T *p, bool live) {
    Quad<T> q;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) q.w[i] = 0;
    if (live) __builtin_memcpy(q.w, p, sizeof(q.w));
    return q;
}
template <typename T> __device__ __forceinline__ void store_quad(T *p, const float (&f)[4]) {
    Quad<T> q;
    if constexpr (sizeof(T) == 2) q.w[0] = round_pair(f[0], f[1]), q.w[1] = round_pair(f[2], f[3]);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) q.w[i] = __float_as_uint(f[i]);
    __builtin_memcpy(p, q.w, sizeof(q.w));
}

template <int G> __device__ __forceinline__ float head_sum(float v) {       // over the G lanes of a head
    if constexpr (G >= 2) v += dpp_move<0xB1>(v);                           // neighbours in pairs
    if constexpr (G >= 4) v += dpp_move<0x4E>(v);                           // pairs of pairs
    if constexpr (G >= 8) v += dpp_move<0x141>(v);                          // mirrored halves of eight lanes
    if constexpr (G >= 16) v += dpp_move<0x140>(v);                         // ... of sixteen
    if constexpr (G >= 32) v = add_rows(v);
    if constexpr (G >= 64) v = add_halves(v);
    return v;
}

// Where the two quads of a lane's piece start, and its angles' first index.
struct Place {
    int first, second, freq;
    bool live, turned;
};
__device__ __forceinline__ Place place_of(const QkArgs &a, int piece) {
    Place p;
    p.live = 8 * piece < a.D;
    p.turned = 8 * piece < a.R;
    const bool halves = p.turned && !a.adjacent;
    p.first = halves ? 4 * piece : 8 * piece;
    p.second = halves ? a.R / 2 + 4 * piece : 8 * piece + 4;
    p.freq = 4 * piece;
    return p;
}
// The cosines and sines of a lane's four angles.  A far position times a frequency has more digits than fp32: the product
// is formed in fp64, in whole turns, and what is left of the last one fits.
__device__ __forceinline__ void angles(const QkArgs &a, const Place &p, long pos, float (&cs)[4], float (&sn)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
    if (!p.turned) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double turns = (double)pos * ((double)a.freq[p.freq + i] * 0.15915494309189533577);
        const float rest = (float)(turns - __builtin_rint(turns));
        sincospif(2.0f * rest, &sn[i], &cs[i]);
    }
}
// (u, v) of each pair turned by the angle (kBack: back)
template <bool kBack> __device__ __forceinline__ void turn(float (&a)[4], float (&b)[4], const float (&cs)[4], const float (&sn)[4], bool adjacent) {
    const auto one = [](float &u, float &v, float c, float s) {
        if constexpr (kBack) s = -s;
        const float x = u;
        u = fmaf(x, c, -v * s);
        v = fmaf(x, s, v * c);
    };
    if (adjacent) {
        one(a[0], a[1], cs[0], sn[0]), one(a[2], a[3], cs[1], sn[1]);
        one(b[0], b[1], cs[2], sn[2]), one(b[2], b[3], cs[3], sn[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) one(a[i], b[i], cs[i], sn[i]);
    }
}
__device__ __forceinline__ float inverse_length(const QkArgs &a, float squares) {
    if (a.norm == 0) return 1.0f;
    return 1.0f / sqrtf((a.norm == LA_QK_RMS ? squares / a.D : squares) + a.eps);
}
__device__ __forceinline__ void weights(const float *w, const Place &p, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = w != nullptr && p.live ? w[(i < 4 ? p.first : p.second - 4) + i] : 1.0f;
}

// Units of work: (token, part), a token's rounds of 64 / G heads dealt to `parts` waves.
template <typename T, int G> __global__ __launch_bounds__(256) void qk_fwd_kernel(const QkArgs a) {
    constexpr int kHeads = kWave / G;
    const int lane = threadIdx.x % kWave, slot = lane / G;
    const Place p = place_of(a, lane % G);
    float wq[8], wk[8];
    weights(a.wq, p, wq);
    weights(a.wk, p, wk);
    const int heads = a.H + a.Hk, rounds = (heads + kHeads - 1) / kHeads;
    const long units = (long)a.B * a.N * a.parts;
    for (long u = (long)blockIdx.x * 4 + threadIdx.x / kWave; u < units; u += (long)gridDim.x * 4) {
        const long token = u / a.parts;
        const int part = (int)(u - token * a.parts), b = (int)(token / a.N), n = (int)(token - (long)b * a.N);
        const bool real = a.lengths == nullptr || n < a.lengths[b];
        float cs[4], sn[4];
        angles(a, p, a.pos != nullptr ? a.pos[token] : n, cs, sn);
        for (int r = part; r < rounds; r += a.parts) {
            const int head = r * kHeads + slot, kh = head - a.H;
            const bool isq = kh < 0, live = p.live && head < heads;
            const T *x = isq ? (const T *)a.q + token * a.ldq + (long)head * a.D : (const T *)a.k + token * a.ldk + (long)kh * a.D;
            const Quad<T> q0 = load_quad<T>(x + p.first, live && real), q1 = load_quad<T>(x + p.second, live && real);
            float f0[4], f1[4], squares = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f0[i] = q0.get(i), f1[i] = q1.get(i);
                squares = fmaf(f0[i], f0[i], squares);
                squares = fmaf(f1[i], f1[i], squares);
            }
            const float inv = inverse_length(a, head_sum<G>(squares));
#pragma unroll
            for (int i = 0; i < 4; ++i) f0[i] *= inv * (isq ? wq[i] : wk[i]), f1[i] *= inv * (isq ? wq[4 + i] : wk[4 + i]);
            turn<false>(f0, f1, cs, sn, a.adjacent);
#pragma unroll
            for (int i = 0; i < 4; ++i) f0[i] = real ? f0[i] : 0.0f, f1[i] = real ? f1[i] : 0.0f;
            T *y = isq ? (T *)a.yq + (token * a.H + head) * a.D : (T *)a.yk + (token * a.Hk + kh) * a.D;
            if (live) {
                store_quad<T>(y + p.first, f0);
                store_quad<T>(y + p.second, f1);
            }
        }
    }
}

// dx = r (g - x r mean(g x r)) with r the inverse length and g = w * (dy turned back); (l2: the sum).  The sums for the
// weights stay in registers over a wave's tokens, those of a workgroup are added in LDS, in a fixed order.
template <typename T, int G> __global__ __launch_bounds__(256) void qk_bwd_kernel(const QkArgs a) {
    constexpr int kHeads = kWave / G;
    const int lane = threadIdx.x % kWave, slot = lane / G;
    const Place p = place_of(a, lane % G);
    float wq[8], wk[8], sq[8], sk[8];
    weights(a.wq, p, wq);
    weights(a.wk, p, wk);
#pragma unroll
    for (int i = 0; i < 8; ++i) sq[i] = sk[i] = 0.0f;
    const int heads = a.H + a.Hk, rounds = (heads + kHeads - 1) / kHeads;
    const long units = (long)a.B * a.N * a.parts;
    for (long u = (long)blockIdx.x * 4 + threadIdx.x / kWave; u < units; u += (long)gridDim.x * 4) {
        const long token = u / a.parts;
        const int part = (int)(u - token * a.parts), b = (int)(token / a.N), n = (int)(token - (long)b * a.N);
        const bool real = a.lengths == nullptr || n < a.lengths[b];
        float cs[4], sn[4];
        angles(a, p, a.pos != nullptr ? a.pos[token] : n, cs, sn);
        for (int r = part; r < rounds; r += a.parts) {
            const int head = r * kHeads + slot, kh = head - a.H;
            const bool isq = kh < 0, live = p.live && head < heads;
            const T *x = isq ? (const T *)a.q + token * a.ldq + (long)head * a.D : (const T *)a.k + token * a.ldk + (long)kh * a.D;
            const long at = isq ? (token * a.H + head) * a.D : (token * a.Hk + kh) * a.D;
            const T *dy = isq ? (const T *)a.dyq + at : (const T *)a.dyk + at;
            const Quad<T> q0 = load_quad<T>(x + p.first, live && real), q1 = load_quad<T>(x + p.second, live && real);
            const Quad<T> d0 = load_quad<T>(dy + p.first, live && real), d1 = load_quad<T>(dy + p.second, live && real);
            float f0[4], f1[4], g0[4], g1[4], squares = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f0[i] = q0.get(i), f1[i] = q1.get(i), g0[i] = d0.get(i), g1[i] = d1.get(i);
                squares = fmaf(f0[i], f0[i], squares);
                squares = fmaf(f1[i], f1[i], squares);
            }
            turn<true>(g0, g1, cs, sn, a.adjacent);
            const float inv = inverse_length(a, head_sum<G>(squares));
            float along = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f0[i] *= inv, f1[i] *= inv;
                // a place without a head has no length either: 0 * inf with eps = 0
                const float s0 = live && real ? g0[i] * f0[i] : 0.0f, s1 = live && real ? g1[i] * f1[i] : 0.0f;
                sq[i] += isq ? s0 : 0.0f, sq[4 + i] += isq ? s1 : 0.0f;
                sk[i] += isq ? 0.0f : s0, sk[4 + i] += isq ? 0.0f : s1;
                g0[i] *= isq ? wq[i] : wk[i], g1[i] *= isq ? wq[4 + i] : wk[4 + i];
                along = fmaf(g0[i], f0[i], along);
                along = fmaf(g1[i], f1[i], along);
            }
            along = head_sum<G>(along);
            along = a.norm == 0 ? 0.0f : a.norm == LA_QK_RMS ? along / a.D : along;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f0[i] = real ? inv * (g0[i] - f0[i] * along) : 0.0f;
                f1[i] = real ? inv * (g1[i] - f1[i] * along) : 0.0f;
            }
            T *dx = isq ? (T *)a.yq + at : (T *)a.yk + at;
            if (live) {
                store_quad<T>(dx + p.first, f0);
                store_quad<T>(dx + p.second, f1);
            }
        }
    }
    if (a.part == nullptr) return;
    __shared__ float red[4][kWave][17];                     // 17: the reading lanes' columns in different banks
#pragma unroll
    for (int i = 0; i < 8; ++i) red[threadIdx.x / kWave][lane][i] = sq[i], red[threadIdx.x / kWave][lane][8 + i] = sk[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * G; i += 256) {
        const int l = i / 16, e = i % 16;
        const Place o = place_of(a, l);
        if (!o.live) continue;
        float v = 0.0f;
        for (int w = 0; w < 4; ++w)
            for (int s = 0; s < kHeads; ++s) v += red[w][s * G + l][e];
        const int in = e % 8;
        a.part[(size_t)blockIdx.x * 2 * a.D + (e < 8 ? 0 : a.D) + (in < 4 ? o.first : o.second - 4) + in] = v;
    }
}

int lanes_of(int D) {
    int g = 1;
    while (8 * g < D) g *= 2;
    return g;
}
}  // namespace

// A token's heads are dealt to several waves where there are fewer tokens than waves have places (256 CUs of 32).
static int parts_of(const QkArgs &a) {
    const int kHeads = kWave / lanes_of(a.D), rounds = (a.H + a.Hk + kHeads - 1) / kHeads;
    const long tokens = (long)a.B * a.N, want = (8192 + tokens - 1) / tokens;
    return (int)(want < rounds ? want : rounds);
}

int qk_groups(const QkArgs &a) {                            // workgroups of the backward, a partial sum of the weights' gradients each
    const long sets = ((long)a.B * a.N * parts_of(a) + 3) / 4;
    return (int)(sets < 1024 ? sets : 1024);
}

hipError_t launch_qk_fwd(QkArgs a, int dtype, hipStream_t s) {
    a.parts = parts_of(a);
    const long sets = ((long)a.B * a.N * a.parts + 3) / 4;
    const unsigned grid = (unsigned)(sets < 65536 ? sets : 65536);
    const int g = lanes_of(a.D);
#define LA_KERNEL(G)                                                          \
    if (g == G) {                                                             \
        if (dtype == 0) qk_fwd_kernel<float, G><<<grid, 256, 0, s>>>(a);      \
        else qk_fwd_kernel<bf16_t, G><<<grid, 256, 0, s>>>(a);                \
    }
    LA_KERNEL(1) LA_KERNEL(2) LA_KERNEL(4) LA_KERNEL(8) LA_KERNEL(16) LA_KERNEL(32) LA_KERNEL(64)
#undef LA_KERNEL
    return hipGetLastError();
}

hipError_t launch_qk_bwd(QkArgs a, int dtype, hipStream_t s) {
    a.parts = parts_of(a);
    const unsigned grid = (unsigned)qk_groups(a);
    const int g = lanes_of(a.D);
#define LA_KERNEL(G)                                                          \
    if (g == G) {                                                             \
        if (dtype == 0) qk_bwd_kernel<float, G><<<grid, 256, 0, s>>>(a);      \
        else qk_bwd_kernel<bf16_t, G><<<grid, 256, 0, s>>>(a);                \
    }
    LA_KERNEL(1) LA_KERNEL(2) LA_KERNEL(4) LA_KERNEL(8) LA_KERNEL(16) LA_KERNEL(32) LA_KERNEL(64)
#undef LA_KERNEL
    return hipGetLastError();
}

}  // namespace la
