// Building blocks of the gated delta rule's kernels: bf16 operands in LDS and in registers.
//
// All products run on v_mfma_f32_16x16x32_bf16: lane (c, g) = (lane % 16, lane / 16) supplies eight contraction indices
// 8g .. 8g + 7 of row (or column) c, and register r of the result holds row 4g + r, column c.  A product's result is an
// operand of the next without leaving its registers: the rows of a pair of result tiles (2s, 2s + 1) are dealt so that lane
// group g has the eight neighbours 32s + 8g .., row i of tile T standing for paired(T, i).
//
// fp32 values are cut into three bf16 parts (exact), elements of bf16 tensors are one part; a product keeps the part
// products down to 2^-16 of its size, so that all of it is exact to about 2^-23.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "la_mixer.h"

namespace la {

__device__ __forceinline__ int paired(int tile, int i) { return 32 * (tile >> 1) + 8 * (i >> 2) + 4 * (tile & 1) + (i & 3); }

template <int P> struct Parts {
    bf16x8_t p[P];
};
template <int PA, int PB> __device__ __forceinline__ f32x4 product(const Parts<PA> &a, const Parts<PB> &b, f32x4 acc) {
#pragma unroll
    for (int s = 2; s >= 0; --s)                              // the small part products first
#pragma unroll
        for (int i = 0; i <= s; ++i)
            if (i < PA && s - i < PB) acc = mfma32_bf16(a.p[i], b.p[s - i], acc);
    return acc;
}
__device__ __forceinline__ Parts<3> cut(f32x4 lo, f32x4 hi) {
    const float x[4] = {lo[0], lo[1], lo[2], lo[3]}, y[4] = {hi[0], hi[1], hi[2], hi[3]};
    const Split3 a = split3(x), b = split3(y);
    return Parts<3>{{cat_parts(a.h, b.h), cat_parts(a.m, b.m), cat_parts(a.l, b.l)}};
}
// A value that a later token of the chunk may have spoiled: its products with masked zeros have to be zeros.
__device__ __forceinline__ f32x4 finite(f32x4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = __builtin_amdgcn_fmed3f(v[r], -3.3e38f, 3.3e38f);
    return v;
}

// ---- matrices of bf16 parts in LDS --------------------------------------------------------------
// Rows of COLS elements in pieces of eight (16 bytes), the pieces of a row exchanged by a function of the row, so that
// 16 lanes that read one piece of 16 rows (also of 16 paired ones) meet all banks.
template <int COLS> __device__ __forceinline__ int mat_at(int row, int piece) {
    const int f = COLS == 32 ? ((row >> 1) & 1) | ((row >> 2) & 2) : (row & 3) | ((row >> 1) & 4);
    return row * COLS + 8 * (piece ^ f);
}
// lane (c, g): eight neighbours of one row
template <int COLS, int P> __device__ __forceinline__ Parts<P> row_operand(const uint16_t *m, int plane, int row, int piece) {
    Parts<P> o;
    const uint16_t *p = m + mat_at<COLS>(row, piece);
#pragma unroll
    for (int i = 0; i < P; ++i) o.p[i] = *reinterpret_cast<const bf16x8_t *>(p + i * plane);
    return o;
}
// Transposed reads: of each group of 16 lanes, lane q supplies the address of four consecutive elements of row q / 4;
// lane i gets element i % 4 of the pieces of lanes i / 4, 4 + i / 4, ..: four rows of one column.
typedef short s16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x2_t read_column(const uint16_t *p) {
    const auto v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)p);
    return __builtin_bit_cast(u32x2_t, v);
}
// lane (c, g): rows row0 + 8g .. 8g + 7 of one column, 16 tile + c or paired(tile, c)
template <int COLS, bool kPaired> __device__ __forceinline__ bf16x8_t column_part(const uint16_t *m, int row0, int tile, int lane) {
    const int q = lane & 15, r = row0 + 8 * (lane >> 4) + (q >> 2);
    const int piece = kPaired ? 4 * (tile >> 1) + (q & 3) : 2 * tile + ((q >> 1) & 1), half = kPaired ? 4 * (tile & 1) : 4 * (q & 1);
    return cat_parts(read_column(m + mat_at<COLS>(r, piece) + half), read_column(m + mat_at<COLS>(r + 4, piece) + half));
}
template <int COLS, bool kPaired, int P> __device__ __forceinline__ Parts<P> column_operand(const uint16_t *m, int plane, int row0, int tile, int lane) {
    Parts<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i) o.p[i] = column_part<COLS, kPaired>(m + i * plane, row0, tile, lane);
    return o;
}

// ---- eight elements of a row on their way to LDS ----------------------------------------------------
template <typename T> struct Eight {
    uint32_t w[2 * sizeof(T)];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};
template <typename T> __device__ __forceinline__ Eight<T> load_eight(const T *p, bool live) {      // at any address
    Eight<T> e;
#pragma unroll
    for (int i = 0; i < (int)(2 * sizeof(T)); ++i) e.w[i] = 0;
    if (live) __builtin_memcpy(e.w, p, sizeof(e.w));
    return e;
}
__device__ __forceinline__ void park_eight(uint16_t *p, int plane, const float (&x)[8]) {
    const Parts<3> c = cut(f32x4{x[0], x[1], x[2], x[3]}, f32x4{x[4], x[5], x[6], x[7]});
#pragma unroll
    for (int i = 0; i < 3; ++i) *reinterpret_cast<bf16x8_t *>(p + i * plane) = c.p[i];
}
template <typename T> __device__ __forceinline__ void park_eight(uint16_t *p, int plane, const Eight<T> &e) {
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x4_t *>(p) = u32x4_t{e.w[0], e.w[1], e.w[2], e.w[3]};
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e.get(i);
        park_eight(p, plane, x);
    }
}

// ---- a chunk --------------------------------------------------------------------------------------
// bf16: 64 tokens, whose elements are one part each.  fp32: 32 tokens of three parts, so that queries, keys and the chunk's
// matrices fit LDS as they do in bf16.
template <typename T> struct Chunk {
    static constexpr int C = sizeof(T) == 2 ? 64 : 32, P = sizeof(T) == 2 ? 1 : 3;
    static constexpr int kTiles = C / 16, kBlocks = C / 32;
    static constexpr int kTri = tri_floats(C), kTriRows = kTri / 32;
};
// row of the 32-column matrix that holds rows `row` of block column `block` (see tri_floats)
template <int C> __device__ __forceinline__ int tri_row(int row, int block) { return block == 0 ? row : C - 32 + row; }

__device__ __forceinline__ float raw_to_f32(const float *p) { return *p; }
__device__ __forceinline__ float raw_to_f32(const bf16_t *p) { return to_f32(*p); }
__device__ __forceinline__ int length_of(const DeltaArgs &a, int b) {
    if (a.lengths == nullptr) return a.N;
    const int n = a.lengths[b];
    return n < 0 ? 0 : n > a.N ? a.N : n;
}

// ---- through the chunks -----------------------------------------------------------------------------
constexpr int kCols = 64;                                    // columns of a workgroup, 16 a wave

// The workgroups of a head's column blocks share its queries, keys and matrices: eight ids apart, they run on one XCD and
// find them in its L2.
__device__ __forceinline__ bool head_and_columns(const DeltaArgs &a, int &bh, int &m0) {
    const int blocks = (a.M + kCols - 1) / kCols, x = blockIdx.x % 8, y = blockIdx.x / 8;
    bh = y / blocks * 8 + x;
    m0 = y % blocks * kCols;
    return bh < a.B * a.H;
}
inline unsigned head_grid(const DeltaArgs &a) { return (unsigned)((a.B * a.H + 7) / 8 * 8 * ((a.M + kCols - 1) / kCols)); }

// K, Q and the chunk-local matrices on their way from memory to LDS.
template <typename T, int D> struct Fetch {
    using Ch = Chunk<T>;
    static constexpr int kTok = Ch::C * D / 8, kTokEach = (kTok + 255) / 256, kTriEach = (2 * Ch::kTri / 8 + 255) / 256;
    Eight<T> k[kTokEach], q[kTokEach];
    Eight<float> tri[kTriEach];
    float gate, beta;
    __device__ __forceinline__ void load(const DeltaArgs &a, long unit, size_t row0, int left, int hk, int h, int tid) {
#pragma unroll
        for (int j = 0; j < kTokEach; ++j) {
            const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
            const bool live = i < kTok && t < left;
            k[j] = load_eight<T>((const T *)a.k + (row0 + t) * a.ldk + (size_t)hk * D + 8 * piece, live);
            q[j] = load_eight<T>((const T *)a.q + (row0 + t) * a.ldq + (size_t)hk * D + 8 * piece, live);
        }
        const float *m = a.tri + unit * 2 * Ch::kTri;
#pragma unroll
        for (int j = 0; j < kTriEach; ++j) tri[j] = load_eight<float>(m + 8 * (tid + 256 * j), tid + 256 * j < 2 * Ch::kTri / 8);
        gate = tid < 2 * Ch::C ? a.gate[unit * 4 * Ch::C + tid] : 0.0f;
        beta = tid < Ch::C && tid < left ? a.beta[(row0 + tid) * a.H + h] : 0.0f;
    }
    __device__ __forceinline__ void park(uint16_t *kS, uint16_t *qS, uint16_t *triS, float *gates, int tid) const {
#pragma unroll
        for (int j = 0; j < kTokEach; ++j) {
            const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
            if (i >= kTok) break;
            park_eight<T>(kS + mat_at<D>(t, piece), Ch::C * D, k[j]);
            park_eight<T>(qS + mat_at<D>(t, piece), Ch::C * D, q[j]);
        }
#pragma unroll
        for (int j = 0; j < kTriEach; ++j) {
            const int i = tid + 256 * j, which = i / (Ch::kTri / 8), at = i % (Ch::kTri / 8);
            if (i >= 2 * Ch::kTri / 8) break;
            park_eight<float>(triS + which * 3 * Ch::kTri + mat_at<32>(at / 4, at % 4), Ch::kTri, tri[j]);
        }
        if (tid < 2 * Ch::C) gates[tid] = gate;
        if (tid < Ch::C) gates[2 * Ch::C + tid] = beta;
    }
};

// 16 columns of a state: tile t, register r holds row paired(t, 4g + r)
template <int D> __device__ __forceinline__ void load_state(const float *p, int M, int g, f32x4 (&S)[D / 16]) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = p == nullptr ? 0.0f : p[(size_t)paired(t, 4 * g + r) * M];
}
template <int D> __device__ __forceinline__ void store_state(float *p, int M, int g, const f32x4 (&S)[D / 16]) {
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[(size_t)paired(t, 4 * g + r) * M] = S[t][r];
}

#define LA_BY_WIDTH(CALL)                                    \
    if (dtype == 0) {                                        \
        if (a.D == 32) CALL(float, 32);                      \
        else if (a.D == 64) CALL(float, 64);                 \
        else CALL(float, 128);                               \
    } else {                                                 \
        if (a.D == 32) CALL(bf16_t, 32);                     \
        else if (a.D == 64) CALL(bf16_t, 64);                \
        else CALL(bf16_t, 128);                              \
    }

}  // namespace la
