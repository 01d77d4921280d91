// Building blocks of the operators around the attention (layer norm, short causal convolution, selective scan)
// and the host-side launchers the C ABI shell calls.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "la_device.h"
#include "la_scan_cut.h"

namespace la {

// ---- rows of elements -------------------------------------------------------------------------
// V consecutive elements of a row as they are in memory.  A row starts wherever the widths before it end, so
// pieces are only aligned to their element; global loads and stores take any address.  Widths that V does
// not divide end in a piece of `valid` < V elements (<= 0: none), which goes element by element.
template <typename T, int V> struct Piece {
    static_assert(V * sizeof(T) >= 4, "whole registers");
    uint32_t w[V * sizeof(T) / 4];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};
template <typename T, int V> __device__ __forceinline__ Piece<T, V> load_piece(const T *p, int valid) {
    Piece<T, V> r;
    if (valid >= V) {
        __builtin_memcpy(r.w, p, sizeof(r.w));
        return r;
    }
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) r.w[i] = 0;
    if (valid <= 0) return r;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i >= valid) break;
        if constexpr (sizeof(T) == 2) r.w[i / 2] |= (uint32_t) reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
        else r.w[i] = reinterpret_cast<const uint32_t *>(p)[i];
    }
    return r;
}
template <typename T, int V> __device__ __forceinline__ Piece<T, V> pack_piece(const float (&f)[V]) {
    Piece<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t b = f32_to_bf16_bits(f[i]);
            if (i & 1) r.w[i / 2] |= b << 16;
            else r.w[i / 2] = b;
        } else {
            r.w[i] = __float_as_uint(f[i]);
        }
    }
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store_piece(T *p, int valid, const Piece<T, V> &r) {
    if (valid >= V) {
        __builtin_memcpy(p, r.w, sizeof(r.w));
        return;
    }
    if (valid <= 0) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i >= valid) break;
        if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2]);
        else reinterpret_cast<uint32_t *>(p)[i] = r.w[i];
    }
}
template <typename T, int V> __device__ __forceinline__ void store_row(T *p, int valid, const float (&f)[V]) {
    store_piece<T, V>(p, valid, pack_piece<T, V>(f));
}
// V fp32 parameters of consecutive channels (zeros behind the last, or without the array)
template <int V> __device__ __forceinline__ void load_params(const float *p, int valid, float (&f)[V], float otherwise = 0.0f) {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = otherwise;
    if (p == nullptr) return;
    if (valid >= V) {
        __builtin_memcpy(f, p, sizeof(f));
        return;
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < valid) f[i] = p[i];
}

// ---- functions ----------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

// log(1 + e) for e in [0, 1]: the logarithm of the rounded sum, and what the sum was rounded by (its slope there,
// 1 / (1 + e), only matters where the remainder does not)
__device__ __forceinline__ float log1p_small(float e) {
    const float u = 1.0f + e;
    return fmaf(__builtin_amdgcn_logf(u), 0.693147180559945f, e - (u - 1.0f));
}
__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.0f) + log1p_small(__expf(-fabsf(v))); }

// ---- sums over lanes ------------------------------------------------------------------------------
typedef unsigned u32x2_pair __attribute__((ext_vector_type(2)));
// over the four groups of 16 lanes, result in all
__device__ __forceinline__ float add_halves(float v) {
    const u32x2_pair r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_rows(float v) {
    const u32x2_pair r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float wave_sum(float v) { return add_halves(add_rows(row_sum16(v))); }

// ---- launchers --------------------------------------------------------------------------------------
// Column sums of part [rows][cols], cols = n[0] + n[1] + n[2]: the first n[0] go to to[0], and so on (NULL: not wanted).
// The rows of a column are added in an order that their number alone decides.
struct SumTargets {
    float *to[3];
    long n[3];
};
hipError_t launch_sum_rows(const float *part, long rows, const SumTargets &out, hipStream_t s);

struct NormArgs {
    const void *x, *r;               // forward: input, residual or NULL; backward: the sum that was normalised, ds or NULL
    const void *dy;
    const float *gamma, *beta, *mean_in, *rstd_in;
    void *y, *s;                     // forward: result, the sum or NULL; backward: dx
    float *mean, *rstd, *part;       // part: [groups][2][E], or with one group straight to
    float *dgamma, *dbeta;
    int rows, E;
    float eps;
};
int norm_groups(int rows, int E, int dtype);    // workgroups of the backward, one partial sum of the weights' gradients each
hipError_t launch_norm_fwd(const NormArgs &a, int dtype, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs &a, int dtype, hipStream_t s);

struct ConvArgs {
    const void *x, *x0, *dy, *dx1;
    const float *w, *bias;
    const int *lengths;
    void *y, *x1, *dx, *dx0;
    float *part;                     // [workgroups][E W + E]: dw and db
    long ldx;
    int B, N, E, W, run, runs;       // runs: pieces of `run` tokens per sequence
    int lpr, groups;                 // lanes per row of a workgroup, workgroups side by side along E
    bool silu;
};
// how a backward cuts its tokens: sets run, runs, lpr, groups; the number of partial sums per channel
long conv_plan_bwd(ConvArgs &a);
hipError_t launch_conv_fwd(ConvArgs a, int dtype, hipStream_t s);
hipError_t launch_conv_bwd(const ConvArgs &a, int dtype, hipStream_t s);
// x [B, E], state [B, W - 1, E] in and out
hipError_t launch_conv_step(const void *x, const float *w, const float *bias, void *state, void *y, int B, int E, int W,
                            bool silu, int dtype, hipStream_t s);

struct ScanArgs {
    const void *x, *dt, *z, *Bt, *Ct, *dy;
    const float *A, *D, *bias, *h0, *dh1;
    const int *lengths;
    void *y, *dx, *ddt, *dz;
    float *h1, *dh0;
    float *keep;                     // [B][tiles][S / 4][E][4]: the states before each tile, or NULL
    float *piece_h;                  // [B][pieces][S / 4][E][4]: of a cut sequence, the state before each piece (backward: the
    float *piece_d;                  //   gradient behind it); [B][pieces][E]: the sum of d of each piece
    float *part_bc;                  // backward: [channel block][B][N][2][S], sums over a block's channels
    float *part;                     //   [B][pieces][E S + 2 E]: dA, dD and ddt_bias of each piece
    void *dB, *dC;
    long ldx, lddt, ldz, ldb, ldc;
    int B, N, E, G, S, tiles, pieces, piece_tiles;
    bool softplus;
};
// pieces that a pass cuts a sequence into (piece_tiles tiles each), from the call's sizes
inline void scan_cut(ScanArgs &a, bool backward) {
    const ScanCut c = scan_cut_of(a.B, a.N, a.E, a.G, a.S, backward);
    a.tiles = c.tiles, a.pieces = c.pieces, a.piece_tiles = c.piece_tiles;
}
// the states before each piece (pieces > 1), then outputs, kept states and the final state; y NULL: kept states only
hipError_t launch_scan_fwd(const ScanArgs &a, int dtype, hipStream_t s);
hipError_t launch_scan_bwd(const ScanArgs &a, int dtype, hipStream_t s);
hipError_t launch_scan_step(const ScanArgs &a, float *h, int dtype, hipStream_t s);

}  // namespace la
