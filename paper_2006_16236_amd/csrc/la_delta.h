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

#include "la_delta_cut.h"
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
// N products with one right operand, a part product of all of them at a time: what follows on each other goes to other results
template <int N, int PA, int PB> __device__ __forceinline__ void products(const Parts<PA> (&a)[N], const Parts<PB> &b, f32x4 (&acc)[N]) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i <= s; ++i)
            if (i < PA && s - i < PB) {
#pragma unroll
                for (int n = 0; n < N; ++n) acc[n] = mfma32_bf16(a[n].p[i], b.p[s - i], acc[n]);
            }
}
// acc[t] += tri[t][s] b[s] over the 32 x 32 blocks on and below the diagonal
template <int N, int S, int PA, int PB> __device__ __forceinline__ void lower_products(const Parts<PA> (&tri)[N][S], const Parts<PB> (&b)[S], f32x4 (&acc)[N]) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 2; k >= 0; --k)
#pragma unroll
            for (int i = 0; i <= k; ++i)
                if (i < PA && k - i < PB) {
#pragma unroll
                    for (int t = 2 * s; t < N; ++t) acc[t] = mfma32_bf16(tri[t][s].p[i], b[s].p[k - i], acc[t]);
                }
}
// the same with the transposed matrix: acc[t] += tri[s][t]^T b[s], blocks s >= t / 2 of block column t / 2
template <int N, int S, int PA, int PB> __device__ __forceinline__ void upper_products(const Parts<PA> (&tri)[N][S], const Parts<PB> (&b)[S], f32x4 (&acc)[N]) {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 2; k >= 0; --k)
#pragma unroll
            for (int i = 0; i <= k; ++i)
                if (i < PA && k - i < PB) {
#pragma unroll
                    for (int t = 0; t < 2 * (s + 1); ++t) acc[t] = mfma32_bf16(tri[t][s].p[i], b[s].p[k - i], acc[t]);
                }
}
// What is written before this point is issued before what is written behind it: the reads of operands that a later product
// takes stay ahead of the products before that.  In the passes (D) not for heads of 32, where the compiler has registers to spare
// and does better alone (8 x 784 x 8 heads of 32 bf16, training step: 106 -> 103 us; heads of 64: the same within 1 %; of 128: spills).
template <int D = 128> __device__ __forceinline__ void in_this_order() {
    if constexpr (D > 32) __builtin_amdgcn_sched_barrier(0);
}
// Between two such points: a matrix instruction (16 cycles of its pipe), then three vector instructions that run beside it, N times.
template <int D, int N> __device__ __forceinline__ void side_by_side() {
    if constexpr (D > 32)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
        }
}
// A value that a later token of the chunk may have spoiled: its products with masked zeros have to be zeros.
__device__ __forceinline__ f32x4 finite(f32x4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = __builtin_amdgcn_fmed3f(v[r], -3.3e38f, 3.3e38f);
    return v;
}

// e^(hi + lo) = 2^(hi log2 e) 2^(what that product's rounding and lo leave), to 2^-22.  Below 2^-126 it is zero.
__device__ __forceinline__ float decay_of(float hi, float lo) {
    constexpr float kLog2e = 1.44269504f, kRest = (float)(1.4426950408889634 - (double)kLog2e), kLn2 = 0.693147181f;
    const float p = hi * kLog2e, rest = fmaf(hi, kLog2e, -p) + fmaf(hi, kRest, lo * kLog2e);
    return __builtin_amdgcn_exp2f(p) * fmaf(rest, kLn2, 1.0f);
}

// ---- matrices of bf16 parts in LDS --------------------------------------------------------------
// Rows of COLS elements in pieces of eight (16 bytes), the pieces of a row exchanged by a function of the row such that a wave's
// reads below take 4.4 cycles, the least for 1 KB (measured; others took 8 or 16): 16-byte reads of one piece of 16 paired
// rows, transposed reads of paired and of neighbouring columns.  kPlain: the same for 16 rows in a run.
template <int COLS, bool kPlain = false> __device__ __forceinline__ int mat_at(int row, int piece) {
    int f;
    if constexpr (kPlain) f = COLS == 128 ? row & 15 : COLS == 64 ? row & 7 : (row >> 1) & 3;
    else f = ((row >> 2) & 3) | (COLS == 128 ? 4 * (row & 3) : COLS == 64 ? 2 * (row & 2) : 0);
    return row * COLS + 8 * (piece ^ f);
}
// lane (c, g): eight neighbours of one row
template <int COLS, int P, bool kPlain = false> __device__ __forceinline__ Parts<P> row_operand(const uint16_t *m, int plane, int row, int piece) {
    Parts<P> o;
    const uint16_t *p = m + mat_at<COLS, kPlain>(row, piece);
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
template <int COLS, bool kPaired, bool kPlain> __device__ __forceinline__ bf16x8_t column_part(const uint16_t *m, int row0, int tile, int lane) {
    const int q = lane & 15, r = row0 + 8 * (lane >> 4) + (q >> 2);
    const int piece = kPaired ? 4 * (tile >> 1) + (q & 3) : 2 * tile + ((q >> 1) & 1), half = kPaired ? 4 * (tile & 1) : 4 * (q & 1);
    return cat_parts(read_column(m + mat_at<COLS, kPlain>(r, piece) + half), read_column(m + mat_at<COLS, kPlain>(r + 4, piece) + half));
}
template <int COLS, bool kPaired, int P, bool kPlain = false> __device__ __forceinline__ Parts<P> column_operand(const uint16_t *m, int plane, int row0, int tile, int lane) {
    Parts<P> o;
#pragma unroll
    for (int i = 0; i < P; ++i) o.p[i] = column_part<COLS, kPaired, kPlain>(m + i * plane, row0, tile, lane);
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
// Values of eight columns.  Each by itself: the remainders of a pair above multiply the other one by zero, and a value that is no finite
// number would spoil its neighbour's column.
template <typename T> __device__ __forceinline__ void park_columns(uint16_t *p, int plane, const Eight<T> &e) {
    if constexpr (sizeof(T) == 2) {
        park_eight<T>(p, plane, e);
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = e.get(i);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            u32x4_t part;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                part[i] = round_pair(x[2 * i], x[2 * i + 1]);
                x[2 * i] -= __uint_as_float(part[i] << 16), x[2 * i + 1] -= __uint_as_float(part[i] & 0xffff0000u);
            }
            *reinterpret_cast<u32x4_t *>(p + k * plane) = part;
        }
    }
}

// The same number, of which the compiler knows nothing: what is computed from it is computed where it is used, instead of ahead of
// a loop for all of its phases in registers that the loop has not got.
__device__ __forceinline__ int here(int n) {
    asm volatile("" : "+v"(n));
    return n;
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

// What a workgroup of a pass does: 64 columns of one piece of one head.
//   kWhole: the pass itself;  kStates: only the state behind the piece (backward: before it);  kTransitions: so too, and with
//   columns of the unit matrix behind those of V.
enum PassKind { kWhole, kStates, kTransitions };
struct Task {
    int bh, b, h, len, piece, first, count;        // chunks first .. first + count - 1
    int m0, cols;
    bool unit;                                     // columns of the unit matrix
    bool start, end;                               // the sequence's first piece, its last one
};
// The workgroups of a head's column blocks share its queries, keys and matrices: eight ids apart, they run on one XCD and
// find them in its L2.  False: nothing to do.
template <PassKind kKind, bool kBack> __device__ __forceinline__ bool task_of(const DeltaArgs &a, int C, int D, Task &t) {
    const int own = (a.M + kCols - 1) / kCols, blocks = own + (kKind == kTransitions ? (D + kCols - 1) / kCols : 0);
    const int pieces = kKind == kWhole ? a.pieces : a.pieces - 1, x = blockIdx.x % 8, y = blockIdx.x / 8, head = y / blocks * 8 + x, block = y % blocks;
    if (head >= a.B * a.H * pieces) return false;
    t.bh = head / pieces, t.piece = head % pieces + (kKind != kWhole && kBack ? 1 : 0);
    t.b = t.bh / a.H, t.h = t.bh % a.H;
    t.unit = block >= own;
    t.m0 = (t.unit ? block - own : block) * kCols;
    const int width = t.unit ? D : a.M;
    t.cols = width - t.m0 < kCols ? width - t.m0 : kCols;
    t.len = length_of(a, t.b);
    const int chunks = (t.len + C - 1) / C, last = chunks > 0 ? (chunks - 1) / a.length : 0;
    t.start = t.piece == 0, t.end = t.piece == last;
    t.first = t.piece * a.length;
    t.count = chunks - t.first < a.length ? chunks - t.first : a.length;
    if (t.piece > last || (kKind != kWhole && !kBack && t.end)) return false;
    return !t.unit || (!t.start && !t.end);        // the first and the last piece start from a state that is there
}
inline unsigned task_grid(const DeltaArgs &a, PassKind kind) {
    const int blocks = (a.M + kCols - 1) / kCols + (kind == kTransitions ? (a.D + kCols - 1) / kCols : 0), pieces = kind == kWhole ? a.pieces : a.pieces - 1;
    return (unsigned)((a.B * a.H * pieces + 7) / 8 * 8 * blocks);
}

// Rows of a tensor as the range check of a buffer descriptor sees them: loads behind the last one's `width` elements give zeros,
// stores there are left out.  The whole offset goes into the lane's own address, which is what is checked.
typedef __amdgpu_buffer_rsrc_t Range;
template <typename T> __device__ __forceinline__ Range range_of(const T *first, int rows, long ld, int width) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(first), 0, rows > 0 ? (int)(((rows - 1) * ld + width) * (long)sizeof(T)) : 0, 0x00020000);
}
template <typename T> __device__ __forceinline__ Eight<T> load_eight(Range r, int byte) {
    Eight<T> e;
    const u32x4_t lo = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, byte, 0, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) e.w[i] = lo[i];
    if constexpr (sizeof(T) == 4) {
        const u32x4_t hi = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, byte + 16, 0, 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) e.w[4 + i] = hi[i];
    }
    return e;
}

// A chunk in LDS, and on its way there: K, Q, a workgroup's columns of V (or dO), the chunk-local matrices, the factors of the
// decay and beta.  Four waves of a workgroup do nothing else: they cut the next chunk's values into parts and write them to the
// other of two buffers while the four others work, one barrier a chunk, and have the one after that on its way from memory.
// kLean: without Q and M, what a pass for states alone needs.
template <typename T, int D, bool kLean = false> struct Chunked {
    using Ch = Chunk<T>;
    static constexpr int kTok = Ch::P * Ch::C * D, kVal = Ch::P * Ch::C * kCols, kTri = 3 * Ch::kTri;
    alignas(16) uint16_t k[kTok], q[kLean ? 8 : kTok], v[kVal], z[kTri], m[kLean ? 8 : kTri];
    alignas(16) float gates[3 * Ch::C];
};
template <typename T, int D, bool kLean> struct Fetch {
    using Ch = Chunk<T>;
    static constexpr int C = Ch::C, kTok = C * D / 8, kTokEach = (kTok + 255) / 256, kVal = C * kCols / 8, kValEach = (kVal + 255) / 256;
    static constexpr int kTri = Ch::kTri / 8, kMats = kLean ? 1 : 2, kTriEach = (kMats * kTri + 255) / 256;
    static_assert(2 * kTri % 256 == 0 && kVal % 256 == 0, "whole turns of 256 threads");
    Eight<T> k[kTokEach], q[kTokEach], v[kValEach];
    Eight<float> tri[kTriEach];
    float gate, beta;
    // left: tokens from this chunk's first to the sequence's end, rows behind it come as zeros; values: at the workgroup's first
    // column, `cols` of them
    __device__ __forceinline__ void load(const DeltaArgs &a, long unit, size_t row0, int left, int hk, int h, const T *values, long ldv, int cols, int tid) {
        const int rows = left < C ? left : C;
        const Range kr = range_of((const T *)a.k + row0 * a.ldk + (size_t)hk * D, rows, a.ldk, D);
        const Range qr = range_of((const T *)a.q + row0 * a.ldq + (size_t)hk * D, rows, a.ldq, D);
        const Range vr = range_of(values + row0 * ldv, rows, ldv, cols);
        const Range br = range_of(a.beta + row0 * a.H + h, rows, a.H, 1);
        constexpr int e = sizeof(T);
#pragma unroll
        for (int j = 0; j < kTokEach; ++j) {
            const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
            k[j] = load_eight<T>(kr, (t * (int)a.ldk + 8 * piece) * e);
            if (!kLean) q[j] = load_eight<T>(qr, (t * (int)a.ldq + 8 * piece) * e);
        }
#pragma unroll
        for (int j = 0; j < kValEach; ++j) {
            const int i = tid + 256 * j, t = i / 8, piece = i % 8;
            v[j] = load_eight<T>(vr, 8 * piece < cols ? (t * (int)ldv + 8 * piece) * e : 0x7fffff00);
        }
        const float *m = a.tri + unit * 2 * Ch::kTri;
#pragma unroll
        for (int j = 0; j < kTriEach; ++j) __builtin_memcpy(tri[j].w, m + 8 * ((tid + 256 * j) % (kMats * kTri)), sizeof(tri[j].w));
        gate = a.gate[unit * 4 * C + tid % (2 * C)];
        beta = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(br, tid * a.H * 4, 0, 0));
    }
    __device__ __forceinline__ void park(Chunked<T, D, kLean> &to, int tid) const {
#pragma unroll
        for (int j = 0; j < kTokEach; ++j) {
            const int i = tid + 256 * j, t = i / (D / 8), piece = i % (D / 8);
            if (kTok % 256 != 0 && i >= kTok) break;
            park_eight<T>(to.k + mat_at<D>(t, piece), C * D, k[j]);
            if (!kLean) park_eight<T>(to.q + mat_at<D>(t, piece), C * D, q[j]);
        }
#pragma unroll
        for (int j = 0; j < kValEach; ++j) {
            const int i = tid + 256 * j;
            park_columns<T>(to.v + mat_at<kCols>(i / 8, i % 8), C * kCols, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kTriEach; ++j) {
            const int i = tid + 256 * j, at = i < kTri ? i : i - kTri;
            if (kMats * kTri % 256 != 0 && i >= kMats * kTri) break;
            park_eight<float>((i < kTri ? to.z : to.m) + mat_at<32>(at / 4, at % 4), Ch::kTri, tri[j]);
        }
        if (tid < 2 * C) to.gates[tid] = gate;
        if (tid < C) to.gates[2 * C + tid] = beta;
    }
};
// The fetching waves of a task, its chunks forwards or backwards.  The others meet the same barriers: one before their first
// chunk, and one behind each.
template <typename T, int D, bool kLean, bool kBack> __device__ __forceinline__ void fetch_chunks(Chunked<T, D, kLean> (&to)[2], const DeltaArgs &a, const Task &task, const T *values,
                                                                                                  long ldv, int tid) {
    constexpr int C = Chunk<T>::C;
    Fetch<T, D, kLean> f;
    const auto load = [&](int i) {
        if (i >= task.count) i = task.count - 1;
        const int chunk = task.first + (kBack ? task.count - 1 - i : i);
        f.load(a, (long)task.bh * a.K + chunk, (size_t)task.b * a.N + (size_t)chunk * C, task.len - chunk * C, task.h / (a.H / a.Hk), task.h,
               values + (size_t)task.h * a.M + task.m0, ldv, task.unit ? 0 : task.cols, tid);
    };
    if (task.count <= 0) return;
    load(0);
    f.park(to[0], tid);
    load(1);
    __syncthreads();
    for (int i = 0; i < task.count; ++i) {
        f.park(to[(i + 1) & 1], tid);
        load(i + 2);
        __syncthreads();
    }
}
// A task's first chunk, by 256 threads that all work on it behind the next barrier
template <typename T, int D> __device__ __forceinline__ void fetch_only(Chunked<T, D> &to, const DeltaArgs &a, const Task &task, const T *values, long ldv, int tid) {
    Fetch<T, D, false> f;
    f.load(a, (long)task.bh * a.K, (size_t)task.b * a.N, task.len, task.h / (a.H / a.Hk), task.h, values + (size_t)task.h * a.M + task.m0, ldv, task.cols, tid);
    f.park(to, tid);
}
// The loads of a state before the first chunk: waited for here, so that the loop need not wait for them with everything else.
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }
// Values in LDS, of P parts: rows row0 .. + 3 of the lane's group, column of this lane, and their sum in fp32.
template <int P> struct Raw4 {
    u32x2_t p[P];
    __device__ __forceinline__ f32x4 sum() const {
        f32x4 v = widen(p[P - 1]);
#pragma unroll
        for (int i = P - 2; i >= 0; --i) v += widen(p[i]);
        return v;
    }
};
template <int COLS, int P, bool kPlain = false> __device__ __forceinline__ Raw4<P> column_values(const uint16_t *m, int plane, int row0, int tile, int lane) {
    const int q = lane & 15, r = row0 + (q >> 2), piece = 2 * tile + ((q >> 1) & 1), half = 4 * (q & 1);
    Raw4<P> v;
#pragma unroll
    for (int i = 0; i < P; ++i) v.p[i] = read_column(m + i * plane + mat_at<COLS, kPlain>(r, piece) + half);
    return v;
}

// 16 columns of a state (zeros without it); `column`: this lane's; tile t, register r holds row paired(t, 4g + r)
template <int D> __device__ __forceinline__ void load_state(const float *state, int column, int M, int g, f32x4 (&S)[D / 16]) {
    const Range r = range_of(state, state == nullptr ? 0 : D, M, M);
    const int lane = (8 * g * M + column) * 4;
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[t][i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, lane + paired(t, i) * M * 4, 0, 0));
}
// The 4 x 4 block of four neighbouring lanes and their four values, transposed: lane 4i + b then has row b of the four columns
// 4i .. + 3, which leave as one 16-byte store instead of four of 4 bytes.
__device__ __forceinline__ f32x4 transpose4(f32x4 v, int lane) {
    const bool odd = lane & 1, high = lane & 2;
    const float a = dpp_move<0xB1>(odd ? v[0] : v[1]), b = dpp_move<0xB1>(odd ? v[2] : v[3]);
    v = f32x4{odd ? a : v[0], odd ? v[1] : a, odd ? b : v[2], odd ? v[3] : b};
    const float c = dpp_move<0x4E>(high ? v[0] : v[2]), d = dpp_move<0x4E>(high ? v[1] : v[3]);
    return f32x4{high ? c : v[0], high ? d : v[1], high ? v[2] : c, high ? v[3] : d};
}
// A wave's 16 x 16 tile of rows `row` + (0 .. 3) per lane group, 16 columns from `column` on, of a row-major matrix
template <typename T> __device__ __forceinline__ void store_tile(Range r, int row, int column, int ld, f32x4 v, int lane) {
    v = transpose4(v, lane);
    const int at = ((row + (lane & 3)) * ld + column + (lane & 12)) * (int)sizeof(T);
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b64(u32x2_t{round_pair(v[0], v[1]), round_pair(v[2], v[3])}, r, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, at, 0, 0);
}
template <int D> __device__ __forceinline__ void store_state(float *state, int column, int M, int lane, const f32x4 (&S)[D / 16]) {
    const Range r = range_of(state, D, M, M);                // M: of the whole state
#pragma unroll
    for (int t = 0; t < D / 16; ++t) store_tile<float>(r, paired(t, 4 * (lane / 16)), column, M, S[t], lane);
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
