// Short causal convolution, one filter of W taps per channel:
//   p_t = bias + sum_k w[k] x_{t-W+1+k},   y_t = p_t sigmoid(p_t)  (or p_t),
// its gradient, and the step for one token of every sequence.
//
// Bound by memory (2 tensors forward, 3 backward).  A thread takes 16 bytes of channels and a run of consecutive
// tokens: the W - 1 rows before a token stay in its registers, so a row is read once per run plus W - 1
// rows at its start, which the neighbouring run has just brought into the caches.  8 x 2048 x 4096 bf16, 4 taps, silu:
// forward 56 us for 268 MB (4.8 TB/s), backward 95 for 403 MB (4.2 TB/s); a copy of 256 MiB has 5.0 TB/s.
#include "la_layer.h"

namespace la {
namespace {

// channels of a thread: 16 bytes, in the backward (whose sums and windows fill the registers) 4 channels
template <typename T> constexpr int kV = 16 / sizeof(T);
constexpr int kVBwd = 4;
constexpr int kAhead = 4;            // rows of a run on their way at a time

// p -> silu(p) and its slope: q = sigmoid(p), p q, q (1 + p (1 - q))
__device__ __forceinline__ float silu_slope(float p, float q) { return q * fmaf(p, 1.0f - q, 1.0f); }

__device__ __forceinline__ int length_of(const int *lengths, int b, int N) {
    return lengths == nullptr ? N : min(max(lengths[b], 0), N);
}

template <int W, int V> struct Filter {
    float w[W][V], bias[V];
    __device__ __forceinline__ Filter(const float *pw, const float *pb, int e, int valid) {
        if (valid >= V) {
            float all[V * W];
            __builtin_memcpy(all, pw + (size_t)e * W, sizeof(all));
#pragma unroll
            for (int i = 0; i < V * W; ++i) w[i % W][i / W] = all[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int k = 0; k < W; ++k) w[k][i] = i < valid ? pw[(size_t)(e + i) * W + k] : 0.0f;
            }
        }
        load_params<V>(pb == nullptr ? nullptr : pb + e, valid, bias);
    }
};

// A thread's V channels from e on: the last ones of a row begin at E - V, and share channels (and results) with the thread
// before.  kNarrow: E < V, `valid` = E of the V are there.
template <bool kNarrow, int V> __device__ __forceinline__ int first_channel(int piece, int E) { return kNarrow ? 0 : min(piece * V, E - V); }
template <bool kNarrow, typename T, int V> __device__ __forceinline__ Piece<T, V> load_row(const T *p, int E) {
    return load_piece<T, V>(p, kNarrow ? E : V);
}
template <bool kNarrow, typename T, int V> __device__ __forceinline__ void store_to(T *p, int E, const float (&f)[V]) {
    store_row<T, V>(p, kNarrow ? E : V, f);
}
template <typename T, int V> __device__ __forceinline__ void keep_if(bool there, Piece<T, V> &p) {
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T) / 4); ++i) p.w[i] = there ? p.w[i] : 0;
}
// Row t of the sequence, t >= -(W - 1): x0 (zeros without it) before token 0, zeros from `end` on.  The address is that of a
// row that is there in any case, and the value is masked: a branch around the load would be waited for.  kInside: the
// caller knows that all rows it asks for are tokens of the sequence.
template <typename T, int W, int V, bool kNarrow> struct Rows {
    const T *x, *x0;                 // at this sequence and channel; x0: its first row
    long ldx;
    int E, end;
    template <bool kInside = false> __device__ __forceinline__ Piece<T, V> at(int t) const {
        if constexpr (kInside) return load_row<kNarrow, T, V>(x + (size_t)t * ldx, E);
        const bool before = t < 0;
        const T *p = before && x0 != nullptr ? x0 + (size_t)(t + W - 1) * E : x + (size_t)max(min(t, end - 1), 0) * ldx;
        Piece<T, V> r = load_row<kNarrow, T, V>(p, E);
        keep_if(before ? x0 != nullptr : t < end, r);
        return r;
    }
};

template <typename T, int W, bool kNarrow> __global__ __launch_bounds__(256) void conv_fwd_kernel(const ConvArgs a) {
    constexpr int V = kV<T>;
    const int pieces = (a.E + V - 1) / V, E = a.E;
    const long id = (long)blockIdx.x * 256 + threadIdx.x;
    const long cut = id / pieces;
    if (cut >= (long)a.B * a.runs) return;
    const int e = first_channel<kNarrow, V>((int)(id - cut * pieces), E), b = (int)(cut / a.runs);
    const int t0 = (int)(cut - (long)b * a.runs) * a.run, t1 = min(t0 + a.run, a.N), len = length_of(a.lengths, b, a.N);
    const Rows<T, W, V, kNarrow> row{(const T *)a.x + (size_t)b * a.N * a.ldx + e,
                                     a.x0 == nullptr ? nullptr : (const T *)a.x0 + (size_t)b * (W - 1) * E + e, a.ldx, E, len};
    const Filter<W, V> f(a.w, a.bias, e, kNarrow ? E : V);
    Piece<T, V> win[W - 1];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) win[k] = row.at(t0 - (W - 1) + k);
    if (a.x1 != nullptr && t0 == 0) {        // the last W - 1 rows of the sequence, rows of x0 among them if it is short
#pragma unroll
        for (int k = 0; k < W - 1; ++k)
            store_piece<T, V>((T *)a.x1 + ((size_t)b * (W - 1) + k) * E + e, kNarrow ? E : V, row.at(len - (W - 1) + k));
    }
    T *y = (T *)a.y + ((size_t)b * a.N + t0) * E + e;
    for (int t = t0; t < t1; t += kAhead) {
        Piece<T, V> next[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) next[j] = row.at(t + j);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float p = f.bias[i];
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    const int at = j + k - (W - 1);      // row of the tap among `win`, `next`
                    p = fmaf(f.w[k][i], at < 0 ? win[at + W - 1].get(i) : next[at].get(i), p);
                }
                const float gate = sigmoid(p);
                o[i] = t + j < len ? (a.silu ? p * gate : p) : 0.0f;
            }
            if (t + j < t1) store_to<kNarrow>(y, E, o);
            y += E;
        }
#pragma unroll
        for (int k = 0; k < W - 1; ++k) win[k] = next[kAhead - (W - 1) + k];
    }
}

// A run [t0, t1) of the gradient: dp_t = dy_t slope(p_t) for t0 <= t < t1 + W - 1 (the last W - 1 belong to the next run
// and are formed again here), dx_t = sum_k w[k] dp_{t+W-1-k}, dw[k] = sum_t dp_t x_{t-W+1+k}, db = sum_t dp_t.
// kInside: all of these tokens are there, and none of them is among the first or last W - 1 of its sequence.
template <typename T, int W, bool kNarrow, bool kInside>
__device__ __forceinline__ void conv_bwd_run(const ConvArgs &a, const Rows<T, W, kVBwd, kNarrow> &row, const Rows<T, W, kVBwd, kNarrow> &grad,
                                             const Filter<W, kVBwd> &f, T *dx, size_t state, int t0, int t1, float (&dw)[W + 1][kVBwd]) {
    constexpr int V = kVBwd;
    const int E = a.E, len = row.end;
    float win[W - 1][V], dp[W][V] = {};      // x_{t-W+1} .. x_{t-1}; dp_{t-W+1} .. dp_t
#pragma unroll
    for (int k = 0; k < W - 1; ++k) {
        const Piece<T, V> p = row.template at<kInside>(t0 - (W - 1) + k);
#pragma unroll
        for (int i = 0; i < V; ++i) win[k][i] = p.get(i);
    }
    for (int t = t0; t < t1 + W - 1; t += kAhead) {
        Piece<T, V> nx[kAhead], nd[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) nx[j] = row.template at<kInside>(t + j), nd[j] = grad.template at<kInside>(t + j);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int now = t + j, out = now - (W - 1);
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x = nx[j].get(i);
                float p = fmaf(f.w[W - 1][i], x, f.bias[i]);
#pragma unroll
                for (int k = 0; k < W - 1; ++k) p = fmaf(f.w[k][i], win[k][i], p);
                const float slope = silu_slope(p, sigmoid(p)), dy = nd[j].get(i);
                // behind the sequence dy is zero, and so is whatever the taps make of its rows
                const float d = a.silu ? dy * slope : dy, mine = now < t1 ? d : 0.0f;
#pragma unroll
                for (int k = 0; k < W - 1; ++k) dp[k][i] = dp[k + 1][i];
                dp[W - 1][i] = d;
#pragma unroll
                for (int k = 0; k < W - 1; ++k) dw[k][i] = fmaf(mine, win[k][i], dw[k][i]);
                dw[W - 1][i] = fmaf(mine, x, dw[W - 1][i]);
                dw[W][i] += mine;
#pragma unroll
                for (int k = 0; k + 1 < W - 1; ++k) win[k][i] = win[k + 1][i];
                win[W - 2][i] = x;
                o[i] = 0.0f;                 // dx_{now - W + 1} = sum_k w[k] dp_{now - k}
#pragma unroll
                for (int k = 0; k < W; ++k) o[i] = fmaf(f.w[k][i], dp[W - 1 - k][i], o[i]);
            }
            T *to = dx + (long)out * E;
            bool store = out >= t0 && out < t1;
            if constexpr (!kInside) {
                // gradient that arrives at the rows handed on: x1 holds rows len - W + 1 .. len - 1
                if (a.dx1 != nullptr && out >= len - (W - 1) && out < len) {
                    const Piece<T, V> g = load_row<kNarrow, T, V>((const T *)a.dx1 + state + (size_t)(out - (len - (W - 1))) * E, E);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] += g.get(i);
                }
                if (t0 == 0 && out < 0) to = (T *)a.dx0 + state + (size_t)(out + W - 1) * E, store = a.dx0 != nullptr;
            }
            if (store) store_to<kNarrow>(to, E, o);
        }
    }
}

// lpr lanes take the pieces of a row side by side, 256 / lpr runs at once; their dw and db are added up in LDS.
template <typename T, int W, bool kNarrow> __global__ __launch_bounds__(256) void conv_bwd_kernel(const ConvArgs a) {
    constexpr int V = kVBwd;
    __shared__ float red[256][V];
    const int E = a.E, lane = threadIdx.x % a.lpr, slot = threadIdx.x / a.lpr, slots = 256 / a.lpr;
    const int piece = (int)(blockIdx.x % a.groups) * a.lpr + lane, pieces = (E + V - 1) / V;
    const long set = blockIdx.x / a.groups, cut = set * slots + slot;
    const int e = first_channel<kNarrow, V>(piece, E);
    float dw[W + 1][V] = {};                 // dw[W]: db
    if (cut < (long)a.B * a.runs && piece < pieces) {
        const int b = (int)(cut / a.runs), t0 = (int)(cut - (long)b * a.runs) * a.run, t1 = min(t0 + a.run, a.N);
        const int len = length_of(a.lengths, b, a.N);
        const Rows<T, W, V, kNarrow> row{(const T *)a.x + (size_t)b * a.N * a.ldx + e,
                                         a.x0 == nullptr ? nullptr : (const T *)a.x0 + (size_t)b * (W - 1) * E + e, a.ldx, E, len};
        const Rows<T, W, V, kNarrow> grad{(const T *)a.dy + (size_t)b * a.N * E + e, nullptr, E, E, min(len, t1 + W - 1)};
        T *dx = (T *)a.dx + (size_t)b * a.N * E + e;
        const size_t state = (size_t)b * (W - 1) * E + e;
        const Filter<W, V> f(a.w, a.bias, e, kNarrow ? E : V);
        // run + W - 1 is a multiple of kAhead: a whole run reads tokens up to t0 + run + W - 2.  One path for all lanes of a wave:
        // where it is cold, fetching the instructions of both takes longer than running one (2 x 133 x 72 bf16: 24 us, not 10),
        // and the masked one alone is 11 % slower where few runs need it (8 x 2048 x 4096 bf16: 106 us, not 95).
        const bool inside = t0 >= W - 1 && t0 + a.run + W - 1 <= len;
        if (__all(inside)) conv_bwd_run<T, W, kNarrow, true>(a, row, grad, f, dx, state, t0, t1, dw);
        else conv_bwd_run<T, W, kNarrow, false>(a, row, grad, f, dx, state, t0, t1, dw);
    }
    if (a.part == nullptr) return;
    for (int k = 0; k <= W; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v = dw[0][i];
#pragma unroll
            for (int m = 1; m <= W; ++m) v = k == m ? dw[m][i] : v;
            red[threadIdx.x][i] = v;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.lpr * V; c += 256) {
            const int its = (int)(blockIdx.x % a.groups) * a.lpr + c / V, from = first_channel<kNarrow, V>(its, E), at = from + c % V;
            // channels of the row's last piece that are the piece before's as well are left to that
            if (its >= pieces || at >= E || at < its * V) continue;
            float v = 0.0f;
            for (int r = 0; r < slots; ++r) v += red[r * a.lpr + c / V][c % V];
            // [E][W] of the taps, then [E] of the bias, as the sums of all workgroups are handed out
            a.part[(size_t)set * E * (W + 1) + (k < W ? (size_t)at * W + k : (size_t)E * W + at)] = v;
        }
    }
}

template <typename T, int W> __global__ __launch_bounds__(256) void conv_step_kernel(const T *x, const float *w, const float *bias, T *state, T *y,
                                                                                   int B, int E, bool silu) {
    constexpr int V = kV<T>;
    const int pieces = (E + V - 1) / V;
    const long id = (long)blockIdx.x * 256 + threadIdx.x;
    if (id >= (long)B * pieces) return;
    const long b = id / pieces;
    const int e = (int)(id - b * pieces) * V, valid = E - e;
    T *rows = state + (size_t)b * (W - 1) * E + e;
    Piece<T, V> r[W];
#pragma unroll
    for (int k = 0; k < W - 1; ++k) r[k] = load_piece<T, V>(rows + (size_t)k * E, valid);
    r[W - 1] = load_piece<T, V>(x + (size_t)b * E + e, valid);
    const Filter<W, V> f(w, bias, e, valid);
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float p = f.bias[i];
#pragma unroll
        for (int k = 0; k < W; ++k) p = fmaf(f.w[k][i], r[k].get(i), p);
        o[i] = silu ? p * sigmoid(p) : p;
    }
    store_row<T, V>(y + (size_t)b * E + e, valid, o);
#pragma unroll
    for (int k = 0; k < W - 1; ++k) store_piece<T, V>(rows + (size_t)k * E, valid, r[k + 1]);
}

#define LA_CONV_DISPATCH(W, dtype, ...)                                                                      \
    do {                                                                                                     \
        if ((dtype) == 0) {                                                                                  \
            using TT = float;                                                                                \
            if ((W) == 2) { constexpr int kW = 2; __VA_ARGS__; }                                             \
            else if ((W) == 3) { constexpr int kW = 3; __VA_ARGS__; }                                        \
            else { constexpr int kW = 4; __VA_ARGS__; }                                                      \
        } else {                                                                                             \
            using TT = bf16_t;                                                                               \
            if ((W) == 2) { constexpr int kW = 2; __VA_ARGS__; }                                             \
            else if ((W) == 3) { constexpr int kW = 3; __VA_ARGS__; }                                        \
            else { constexpr int kW = 4; __VA_ARGS__; }                                                      \
        }                                                                                                    \
    } while (0)

int pieces_of(int E, int dtype) { return dtype == 0 ? (E + 3) / 4 : (E + 7) / 8; }

}  // namespace

hipError_t launch_conv_fwd(ConvArgs a, int dtype, hipStream_t s) {
    const long pieces = pieces_of(a.E, dtype);
    // 16 tokens a run; shorter ones where those are too few threads for the machine
    a.run = 16;
    while (a.run > 4 && a.B * pieces * ((a.N + a.run - 1) / a.run) < 256 * 1024) a.run /= 2;
    a.runs = (a.N + a.run - 1) / a.run;
    const long threads = (long)a.B * a.runs * pieces;
    const unsigned grid = (unsigned)((threads + 255) / 256);
    LA_CONV_DISPATCH(a.W, dtype, {
        if (a.E < kV<TT>) conv_fwd_kernel<TT, kW, true><<<grid, 256, 0, s>>>(a);
        else conv_fwd_kernel<TT, kW, false><<<grid, 256, 0, s>>>(a);
    });
    return hipGetLastError();
}

long conv_plan_bwd(ConvArgs &a) {
    const int pieces = (a.E + kVBwd - 1) / kVBwd;
    a.lpr = 64;
    while (a.lpr / 2 >= pieces && a.lpr > 1) a.lpr /= 2;
    a.groups = (pieces + a.lpr - 1) / a.lpr;
    // 32 steps a run, W - 1 of them on the next run's tokens (64: 107 instead of 95 us at 8 x 2048 x 4096 bf16); 16 or 8
    // where those are too few threads (3 x 2531 x 1001 fp32: 16 take 29 us, 8 take 36; 2 x 133 x 72 bf16: 15 and 12)
    int steps = 32;
    const auto threads = [&] { return (long)a.B * pieces * ((a.N + steps - a.W) / (steps - a.W + 1)); };
    if (threads() < 192 * 1024) steps = 16;
    if (threads() < 16 * 1024) steps = 8;
    a.run = steps - (a.W - 1);
    a.runs = (a.N + a.run - 1) / a.run;
    const long cuts = (long)a.B * a.runs, slots = 256 / a.lpr;
    return (cuts + slots - 1) / slots;
}

hipError_t launch_conv_bwd(const ConvArgs &a, int dtype, hipStream_t s) {
    ConvArgs p = a;
    const long sets = conv_plan_bwd(p);
    const unsigned grid = (unsigned)(sets * p.groups);
    LA_CONV_DISPATCH(a.W, dtype, {
        if (a.E < kVBwd) conv_bwd_kernel<TT, kW, true><<<grid, 256, 0, s>>>(p);
        else conv_bwd_kernel<TT, kW, false><<<grid, 256, 0, s>>>(p);
    });
    return hipGetLastError();
}

hipError_t launch_conv_step(const void *x, const float *w, const float *bias, void *state, void *y, int B, int E, int W,
                            bool silu, int dtype, hipStream_t s) {
    const long threads = (long)B * pieces_of(E, dtype);
    LA_CONV_DISPATCH(W, dtype, conv_step_kernel<TT, kW><<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(
        (const TT *)x, w, bias, (TT *)state, (TT *)y, B, E, silu));
    return hipGetLastError();
}

}  // namespace la
