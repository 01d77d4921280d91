// Layer norm over rows of E elements, y = (s - mean) * rstd * gamma + beta with s = x + r, and its gradient.
//
// Bound by memory: forward 2 tensors (4 with a residual and its sum), backward 3 (4).  A row lives in the
// registers of the lanes that share it, so that each element is read once: mean, then the sum of squares around it
// (two passes over registers, no cancellation as in E[x^2] - mean^2), then the result.  16 or 32 lanes share a row
// of as many 16-byte pieces, 64 one of up to 1024 elements, 256 (backward: 128 up to 2048) up to 8192, 1024 (backward 512) up to
// 16384.  With a residual, bf16, 16384 x 4096: forward 96 us, backward 117, 5.6 and 4.6 TB/s of 4 tensors each, where a copy
// of 256 MiB has 5.0; 16384 x 2048: 52 and 54 us.
#include "la_layer.h"

namespace la {
namespace {

constexpr int kSumSlices = 16;
constexpr int kBwdThreads = 512;
// Workgroups of a launch; more rows go round again (more columns of the sums in another launch).  A workgroup of 1024 lanes that keeps
// its weights for several rows is 6 % faster than one a row, one of 256 is 5 % slower.
constexpr long kMaxGrid = 1 << 20, kWideGrid = 2048;

__global__ __launch_bounds__(1024) void sum_rows_kernel(const float *__restrict__ part, long rows, const SumTargets out, long first) {
    __shared__ float red[kSumSlices][kWave];
    const int lane = threadIdx.x % kWave, slice = threadIdx.x / kWave;
    const long cols = out.n[0] + out.n[1] + out.n[2], c = first + (long)blockIdx.x * kWave + lane;
    float v = 0.0f;
    if (c < cols) {
        long r = slice;
        for (; r + 3 * kSumSlices < rows; r += 4 * kSumSlices) {        // four loads on their way at a time
            float t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = part[(r + i * kSumSlices) * cols + c];
#pragma unroll
            for (int i = 0; i < 4; ++i) v += t[i];
        }
        for (; r < rows; r += kSumSlices) v += part[r * cols + c];
    }
    red[slice][lane] = v;
    __syncthreads();
    if (slice != 0 || c >= cols) return;
#pragma unroll
    for (int i = 1; i < kSumSlices; ++i) v += red[i][lane];
    const int k = c < out.n[0] ? 0 : c < out.n[0] + out.n[1] ? 1 : 2;
    const long at = c - (k > 0 ? out.n[0] : 0) - (k > 1 ? out.n[1] : 0);
    float *to = k == 0 ? out.to[0] : k == 1 ? out.to[1] : out.to[2];
    if (to != nullptr) to[at] = v;
}

// sum over the TPR lanes that share a row; `red`: one slot per wave of the workgroup
template <int TPR> __device__ __forceinline__ float lanes_sum(float v) {        // within a wave
    if constexpr (TPR == 16) return row_sum16(v);
    else if constexpr (TPR == 32) return add_rows(row_sum16(v));
    else return wave_sum(v);
}
template <int TPR> __device__ __forceinline__ float row_sum(float v, float *red) {
    v = lanes_sum<TPR>(v);
    if constexpr (TPR > kWave) {
        const int wave = threadIdx.x / kWave, first = wave / (TPR / kWave) * (TPR / kWave);
        __syncthreads();
        if (threadIdx.x % kWave == 0) red[wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / kWave; ++i) v += red[first + i];
    }
    return v;
}

// TPR lanes per row, NV pieces of V elements per lane (piece j of lane l starts at element (j * TPR + l) * V)
template <typename T, int TPR, int NV> __global__ __launch_bounds__(TPR > 256 ? TPR : 256) void norm_fwd_kernel(const NormArgs a) {
    constexpr int V = 16 / sizeof(T), kThreads = TPR > 256 ? TPR : 256, kRows = kThreads / TPR;
    // all loads of a row on their way first (8192 x 8192 bf16: 111 -> 100 us), or a piece and its residual at a time, whose sum is
    // stored meanwhile (2048 x 1024 fp32: 8.7 us, not 10.0; 4096 x 16384 bf16: 104, not 108)
    constexpr bool kAhead = sizeof(T) == 2 && TPR <= 256;
    __shared__ float red[kThreads / kWave];
    const int E = a.E, l = threadIdx.x % TPR;
    float g[NV][V], b[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int e = (j * TPR + l) * V;
        load_params<V>(a.gamma == nullptr ? nullptr : a.gamma + e, E - e, g[j], 1.0f);
        load_params<V>(a.beta == nullptr ? nullptr : a.beta + e, E - e, b[j]);
    }
    for (long first = (long)blockIdx.x * kRows; first < a.rows; first += (long)gridDim.x * kRows) {
        const long row = first + threadIdx.x / TPR;
        const bool live = row < a.rows;          // all lanes meet in row_sum
        const size_t at = (size_t)row * E;
        Piece<T, V> p[NV], q[NV];
        const auto load = [&](int j) {
            const int e = (j * TPR + l) * V, valid = live ? E - e : 0;
            p[j] = load_piece<T, V>((const T *)a.x + at + e, valid);
            if (a.r != nullptr) q[j] = load_piece<T, V>((const T *)a.r + at + e, valid);
        };
        if constexpr (kAhead) {
#pragma unroll
            for (int j = 0; j < NV; ++j) load(j);
        }
        float f[NV][V];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (!kAhead) load(j);
            if (a.r != nullptr) {
                float t[V];
#pragma unroll
                for (int i = 0; i < V; ++i) t[i] = p[j].get(i) + q[j].get(i);
                // the stored sum is what the backward (and the next layer) reads: it is what is normalised
                p[j] = pack_piece<T, V>(t);
                const int e = (j * TPR + l) * V;
                if (a.s != nullptr) store_piece<T, V>((T *)a.s + at + e, live ? E - e : 0, p[j]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum += f[j][i] = p[j].get(i);
        }
        const float mean = row_sum<TPR>(sum, red) / E;
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[j][i] -= mean;
                if ((j * TPR + l) * V + i < E) sq = fmaf(f[j][i], f[j][i], sq);
            }
        }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(sq, red) / E + a.eps);
        if (l == 0 && live) {
            if (a.mean != nullptr) a.mean[row] = mean;
            if (a.rstd != nullptr) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (j * TPR + l) * V;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = fmaf(f[j][i] * rstd, g[j][i], b[j][i]);
            store_row<T, V>((T *)a.y + at + e, live ? E - e : 0, o);
        }
    }
}

// xhat = (s - mean) rstd, g = dy gamma, dx = rstd (g - mean(g) - xhat mean(g xhat)) + ds; a workgroup takes every
// gridDim-th set of rows and keeps its part of dgamma = sum dy xhat, dbeta = sum dy in registers, which take as much room as
// the row: 16 elements a lane up to 2048 (16384 x 2048 bf16: 52 us, 32 a lane 55, and 8 a lane 55).
template <typename T, int TPR, int NV> __global__ __launch_bounds__(kBwdThreads) void norm_bwd_kernel(const NormArgs a) {
    constexpr int V = 16 / sizeof(T), kRows = kBwdThreads / TPR, kHalf = kRows > 1 ? kRows / 2 : 1, kCols = NV * V;
    // all of ds on its way first (8192 x 8192 fp32: 231 -> 211 us; bf16 131 -> 121), but where that takes the registers of a
    // wave more (8192 x 1536 fp32: 36 us, not 41)
    constexpr bool kAhead = sizeof(T) == 2 || kCols > 16;
    __shared__ float red[2 * kBwdThreads / kWave];
    __shared__ float part[kHalf][kCols][TPR];
    const int E = a.E, l = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float dg[NV][V] = {}, db[NV][V] = {};
    for (long first = (long)blockIdx.x * kRows; first < a.rows; first += (long)gridDim.x * kRows) {
        const long row = first + slot;
        const bool live = row < a.rows;
        const float mean = live ? a.mean_in[row] : 0.0f, rstd = live ? a.rstd_in[row] : 0.0f;
        Piece<T, V> s[NV], d[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (j * TPR + l) * V, valid = live ? E - e : 0;
            s[j] = load_piece<T, V>((const T *)a.x + (size_t)row * E + e, valid);
            d[j] = load_piece<T, V>((const T *)a.dy + (size_t)row * E + e, valid);
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float gamma[V];
            load_params<V>(a.gamma == nullptr ? nullptr : a.gamma + (j * TPR + l) * V, E - (j * TPR + l) * V, gamma, 1.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xhat = (s[j].get(i) - mean) * rstd, dy = d[j].get(i), g = dy * gamma[i];
                s1 += g;
                s2 = fmaf(g, xhat, s2);
                dg[j][i] = fmaf(dy, xhat, dg[j][i]);
                db[j][i] += dy;
            }
        }
        s1 = lanes_sum<TPR>(s1), s2 = lanes_sum<TPR>(s2);
        if constexpr (TPR > kWave) {
            const int wave = threadIdx.x / kWave, w0 = wave / (TPR / kWave) * (TPR / kWave);
            __syncthreads();
            if (threadIdx.x % kWave == 0) red[2 * wave] = s1, red[2 * wave + 1] = s2;
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < TPR / kWave; ++i) s1 += red[2 * (w0 + i)], s2 += red[2 * (w0 + i) + 1];
        }
        s1 /= E, s2 /= E;
        const size_t at = (size_t)row * E;
        Piece<T, V> ds[NV] = {};
        const auto load = [&](int j) {
            const int e = (j * TPR + l) * V;
            if (a.r != nullptr) ds[j] = load_piece<T, V>((const T *)a.r + at + e, live ? E - e : 0);
        };
        if constexpr (kAhead) {
#pragma unroll
            for (int j = 0; j < NV; ++j) load(j);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int e = (j * TPR + l) * V;
            if constexpr (!kAhead) load(j);
            float gamma[V], o[V];
            load_params<V>(a.gamma == nullptr ? nullptr : a.gamma + e, E - e, gamma, 1.0f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xhat = (s[j].get(i) - mean) * rstd, g = d[j].get(i) * gamma[i];
                o[i] = fmaf(rstd, g - fmaf(xhat, s2, s1), ds[j].get(i));
            }
            store_row<T, V>((T *)a.y + at + e, live ? E - e : 0, o);
        }
    }
    if (a.part == nullptr) return;
    // the row slots' sums, halving their number with every step
    auto gather = [&](float(&v)[NV][V]) {
#pragma unroll
        for (int half = kRows / 2; half >= 1; half /= 2) {
            __syncthreads();
            if (slot >= half && slot < 2 * half) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) part[slot - half][c][l] = v[c / V][c % V];
            }
            __syncthreads();
            if (slot < half) {
#pragma unroll
                for (int c = 0; c < kCols; ++c) v[c / V][c % V] += part[slot][c][l];
            }
        }
    };
    gather(dg);
    gather(db);
    if (slot != 0) return;
    float *pg = a.part + (size_t)blockIdx.x * 2 * E, *pb = pg + E;
    if (gridDim.x == 1) pg = a.dgamma, pb = a.dbeta;                     // a part that is the whole
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int e = (j * TPR + l) * V;
        if (pg != nullptr) store_row<float, V>(pg + e, E - e, dg[j]);
        if (pb != nullptr) store_row<float, V>(pb + e, E - e, db[j]);
    }
}

// forward: beyond 8192 elements 16 a lane again (4096 x 16384 bf16: 512 lanes of 32 take 137 us, 1024 of 16 take 106)
int lanes_of(int E, int dtype) {
    const int pieces = dtype == 0 ? (E + 3) / 4 : (E + 7) / 8;
    return pieces <= 16 ? 16 : pieces <= 32 ? 32 : E <= 1024 ? 64 : E <= 8192 ? 256 : 1024;
}
int lanes_of_bwd(int E, int dtype) {
    const int pieces = dtype == 0 ? (E + 3) / 4 : (E + 7) / 8;
    return pieces <= 16 ? 16 : pieces <= 32 ? 32 : E <= 1024 ? 64 : E <= 2048 ? 128 : E <= 8192 ? 256 : 512;
}

}  // namespace

hipError_t launch_sum_rows(const float *part, long rows, const SumTargets &out, hipStream_t s) {
    const long cols = out.n[0] + out.n[1] + out.n[2];
    for (long first = 0; first < cols; first += kMaxGrid * kWave) {       // one launch; 2^32 lanes and more would be none
        const long blocks = (cols - first + kWave - 1) / kWave;
        sum_rows_kernel<<<(unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid), 1024, 0, s>>>(part, rows, out, first);
    }
    return hipGetLastError();
}

// Two workgroups a compute unit, or one where more than 16 elements a lane leave room for no more (16384 x 4096 bf16, 16 a
// lane: 113 us with 512 workgroups, 140 with 256; with 32 a lane 62 and 55 at 16384 x 2048).
int norm_groups(int rows, int E, int dtype) {
    const int tpr = lanes_of_bwd(E, dtype), per = kBwdThreads / tpr, most = E > 16 * tpr ? 256 : 512;
    const long sets = ((long)rows + per - 1) / per, turns = (sets + most - 1) / most;      // equal shares
    return (int)((sets + turns - 1) / turns);
}

// pieces of 16 bytes a lane has of a row that `tpr` lanes share
static int pieces_of(int E, int tpr, int dtype) {
    const int v = tpr * (dtype == 0 ? 4 : 8);
    return (E + v - 1) / v;
}

hipError_t launch_norm_fwd(const NormArgs &a, int dtype, hipStream_t s) {
#define LA_KERNEL(T, TPR, NV)                                                                                        \
    do {                                                                                                             \
        constexpr int threads = TPR > 256 ? TPR : 256, per = threads / TPR;                                          \
        constexpr long most = TPR > 256 ? kWideGrid : kMaxGrid;                                                      \
        const long sets = ((long)a.rows + per - 1) / per;                                                            \
        norm_fwd_kernel<T, TPR, NV><<<(unsigned)(sets < most ? sets : most), threads, 0, s>>>(a);                    \
    } while (0)
    const int tpr = lanes_of(a.E, dtype), nv = pieces_of(a.E, tpr, dtype);
    if (dtype == 0) {
        if (tpr == 16) {
            LA_KERNEL(float, 16, 1);
        } else if (tpr == 32) {
            LA_KERNEL(float, 32, 1);
        } else if (tpr == 64) {
            if (nv <= 1) LA_KERNEL(float, 64, 1);
            else if (nv == 2) LA_KERNEL(float, 64, 2);
            else LA_KERNEL(float, 64, 4);
        } else if (tpr == 256) {
            if (nv <= 2) LA_KERNEL(float, 256, 2);
            else if (nv <= 4) LA_KERNEL(float, 256, 4);
            else LA_KERNEL(float, 256, 8);
        } else {
            LA_KERNEL(float, 1024, 4);
        }
    } else {
        if (tpr == 16) {
            LA_KERNEL(bf16_t, 16, 1);
        } else if (tpr == 32) {
            LA_KERNEL(bf16_t, 32, 1);
        } else if (tpr == 64) {
            if (nv <= 1) LA_KERNEL(bf16_t, 64, 1);
            else LA_KERNEL(bf16_t, 64, 2);
        } else if (tpr == 256) {
            if (nv <= 1) LA_KERNEL(bf16_t, 256, 1);
            else if (nv == 2) LA_KERNEL(bf16_t, 256, 2);
            else LA_KERNEL(bf16_t, 256, 4);
        } else {
            LA_KERNEL(bf16_t, 1024, 2);
        }
    }
#undef LA_KERNEL
    return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormArgs &a, int dtype, hipStream_t s) {
#define LA_KERNEL(T, TPR, NV) norm_bwd_kernel<T, TPR, NV><<<groups, kBwdThreads, 0, s>>>(a)
    const int groups = norm_groups(a.rows, a.E, dtype), tpr = lanes_of_bwd(a.E, dtype), nv = pieces_of(a.E, tpr, dtype);
    if (dtype == 0) {
        if (tpr == 16) {
            LA_KERNEL(float, 16, 1);
        } else if (tpr == 32) {
            LA_KERNEL(float, 32, 1);
        } else if (tpr == 64) {
            if (nv <= 1) LA_KERNEL(float, 64, 1);
            else if (nv == 2) LA_KERNEL(float, 64, 2);
            else LA_KERNEL(float, 64, 4);
        } else if (tpr == 128) {
            LA_KERNEL(float, 128, 4);
        } else if (tpr == 256) {
            if (nv <= 4) LA_KERNEL(float, 256, 4);
            else LA_KERNEL(float, 256, 8);
        } else {
            LA_KERNEL(float, 512, 8);
        }
    } else {
        if (tpr == 16) {
            LA_KERNEL(bf16_t, 16, 1);
        } else if (tpr == 32) {
            LA_KERNEL(bf16_t, 32, 1);
        } else if (tpr == 64) {
            if (nv <= 1) LA_KERNEL(bf16_t, 64, 1);
            else LA_KERNEL(bf16_t, 64, 2);
        } else if (tpr == 128) {
            LA_KERNEL(bf16_t, 128, 2);
        } else if (tpr == 256) {
            if (nv == 2) LA_KERNEL(bf16_t, 256, 2);
            else LA_KERNEL(bf16_t, 256, 4);
        } else {
            LA_KERNEL(bf16_t, 512, 4);
        }
    }
#undef LA_KERNEL
    return hipGetLastError();
}

}  // namespace la
