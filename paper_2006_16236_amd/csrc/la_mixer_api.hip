// The C ABI of the head norm with rotation and of the gated delta rule: argument checks, workspace carving and launches.
#include <math.h>

#include "la_checks.h"
#include "la_mixer.h"

namespace {
using namespace la_check;

int esize_of(la_dtype t) { return t == LA_BF16 ? 2 : 4; }
bool known(la_dtype t) { return t == LA_F32 || t == LA_BF16; }
// bytes from the first element of `rows` strided rows to behind the last one's `width` elements
size_t span(size_t rows, size_t ld, size_t width, la_dtype t) { return ((rows - 1) * ld + width) * esize_of(t); }
size_t span_of(const void *p, size_t bytes) { return p == nullptr ? 0 : bytes; }
template <typename... Ps> bool any_misaligned(Ps... p) { return (misaligned(p) || ...); }
template <typename... Ps> bool any_null(Ps... p) { return ((p == nullptr) || ...); }

constexpr int kMostInt = 1 << 30;                            // tokens are counted in int, a chunk ahead of the last one
constexpr double kMostElements = 68719476736.0;              // 2^36
constexpr int kMostApart = 1 << 23;                          // elements between tokens: a chunk is addressed with 31 bits of bytes
constexpr double kMostUnits = 8388608.0;                     // 2^23 workgroups of up to 512 threads are one launch

// ---- head norm and rotation -------------------------------------------------------------------------
constexpr int kMaxHead = 512;

int qk_sizes(int B, int N, int H, int Hk, int D, int R, int flags, la_dtype t) {
    if (!known(t) || (flags & ~(LA_QK_RMS | LA_QK_L2 | LA_QK_ADJACENT)) != 0 || (flags & (LA_QK_RMS | LA_QK_L2)) == (LA_QK_RMS | LA_QK_L2))
        return LA_ERR_UNSUPPORTED;
    if (B < 1 || N < 1 || H < 1 || Hk < 0 || D < 1 || R < 0 || R > D || N > kMostInt) return LA_ERR_SHAPE;
    if (D > kMaxHead || D % 8 != 0 || R % 8 != 0) return LA_ERR_UNSUPPORTED;
    if (((double)H + Hk) * D > kMostInt || (double)B * N * ((double)H + Hk) * D >= kMostElements) return LA_ERR_SHAPE;
    return LA_OK;
}
la::QkArgs qk_args(int B, int N, int H, int Hk, int D, int R, int flags, float eps) {
    la::QkArgs a{};
    a.B = B, a.N = N, a.H = H, a.Hk = Hk, a.D = D, a.R = R, a.eps = eps;
    a.norm = flags & (LA_QK_RMS | LA_QK_L2), a.adjacent = (flags & LA_QK_ADJACENT) != 0;
    return a;
}
size_t qk_bytes(const la::QkArgs &a) { return align256((size_t)la::qk_groups(a) * 2 * a.D * sizeof(float)); }

// ---- gated delta rule ---------------------------------------------------------------------------------
int delta_sizes(int B, int N, int H, int Hk, int D, int M, la_dtype t, int flags) {
    if (!known(t) || (flags & ~LA_DELTA_KEEP) != 0) return LA_ERR_UNSUPPORTED;
    if (B < 1 || N < 1 || H < 1 || Hk < 1 || D < 1 || M < 1 || H % Hk != 0 || N > kMostInt) return LA_ERR_SHAPE;
    if (!(D == 32 || D == 64 || D == 128) || M % 16 != 0 || M > 512) return LA_ERR_UNSUPPORTED;
    const int C = la::delta_chunk(t);
    if ((double)H * M > kMostApart || (double)Hk * D > kMostApart || (double)B * N * H * (M > D ? M : D) >= kMostElements) return LA_ERR_SHAPE;
    if (((double)B * H + 8) * ((N + (double)C - 1) / C) >= kMostUnits || ((double)B * H + 8) * ((M + 63) / 64) >= kMostUnits) return LA_ERR_SHAPE;
    // a sequence is cut only where its pieces are at most 64 and there are few of them: their grids are far smaller
    return LA_OK;
}
bool bad_apart(int ld, int width) { return ld < width || ld > kMostApart; }
struct Delta {
    la::DeltaArgs a{};
    size_t tri, gate, rows, state, pieces, transitions;
    Delta(int B, int N, int H, int Hk, int D, int M, float scale, la_dtype t) {
        const int C = la::delta_chunk(t);
        a.B = B, a.N = N, a.H = H, a.Hk = Hk, a.D = D, a.M = M, a.scale = scale;
        a.K = (N - 1) / C + 1;
        const size_t units = (size_t)B * H * a.K;
        tri = units * 2 * la::tri_floats(C) * sizeof(float);
        gate = units * 4 * C * sizeof(float);
        rows = units * C * M * sizeof(float);
        state = units * D * M * sizeof(float);
        const la::DeltaCut cut = la::delta_cut_of((long)B * H, D, M, a.K, esize_of(t));
        a.pieces = cut.pieces, a.length = cut.length;
        const size_t cuts = cut.pieces > 1 ? (size_t)B * H * cut.pieces : 0;
        pieces = cuts * D * M * sizeof(float), transitions = cuts * D * D * sizeof(float);
    }
    size_t fwd_bytes(bool keep) const {
        return align256(tri) + align256(gate) + align256(pieces) + align256(transitions) + (keep ? align256(rows) + align256(state) : 0);
    }
    size_t bwd_bytes(bool given) const { return align256(rows) + align256(state) + align256(pieces) + (given ? 0 : fwd_bytes(true)); }
    void carve_fwd(Carver &cv, bool keep) {
        a.piece_state = static_cast<float *>(cv.take(pieces)), a.transition = static_cast<float *>(cv.take(transitions));
        a.tri = static_cast<float *>(cv.take(tri)), a.gate = static_cast<float *>(cv.take(gate));
        if (keep) a.miss = static_cast<float *>(cv.take(rows)), a.state = static_cast<float *>(cv.take(state));
    }
};
}  // namespace

extern "C" {

int la_qk_fwd(const void *q, int ldq, const void *k, int ldk, const float *wq, const float *wk, const float *freq, const int *pos,
              const int *lengths, void *yq, void *yk, int B, int N, int H, int Hk, int D, int R, int flags, float eps, la_dtype t, void *stream) {
    if (any_null(q, yq) || (Hk > 0 && any_null(k, yk)) || (R > 0 && freq == nullptr)) return LA_ERR_NULL;
    const int st = qk_sizes(B, N, H, Hk, D, R, flags, t);
    if (st != LA_OK) return st;
    if (!(eps >= 0.0f) || !isfinite(eps) || ldq < H * D || (Hk > 0 && ldk < Hk * D)) return LA_ERR_SHAPE;
    if (any_misaligned(q, k, wq, wk, freq, pos, lengths, yq, yk)) return LA_ERR_ALIGN;
    const size_t T = (size_t)B * N, w = (size_t)D * 4;
    const Span outs[] = {{yq, span(T, H * D, H * D, t)}, {yk, Hk > 0 ? span(T, Hk * D, Hk * D, t) : 0}};
    const Span ins[] = {{q, span(T, ldq, H * D, t)}, {k, Hk > 0 ? span(T, ldk, Hk * D, t) : 0}, {wq, span_of(wq, w)}, {wk, span_of(wk, w)},
                        {freq, span_of(freq, (size_t)R * 2)}, {pos, span_of(pos, T * 4)}, {lengths, span_of(lengths, (size_t)B * 4)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::QkArgs a = qk_args(B, N, H, Hk, D, R, flags, eps);
    a.q = q, a.k = k, a.wq = wq, a.wk = wk, a.freq = freq, a.pos = pos, a.lengths = lengths, a.yq = yq, a.yk = yk;
    a.ldq = ldq, a.ldk = ldk;
    return hip_status(la::launch_qk_fwd(a, t, static_cast<hipStream_t>(stream)));
}

size_t la_qk_bwd_workspace(int B, int N, int H, int Hk, int D, la_dtype t) {
    if (qk_sizes(B, N, H, Hk, D, 0, 0, t) != LA_OK) return 0;
    return qk_bytes(qk_args(B, N, H, Hk, D, 0, 0, 0.0f));
}

int la_qk_bwd(const void *q, int ldq, const void *k, int ldk, const float *wq, const float *wk, const float *freq, const int *pos,
              const int *lengths, const void *dyq, const void *dyk, void *dq, void *dk, float *dwq, float *dwk, int B, int N, int H, int Hk,
              int D, int R, int flags, float eps, la_dtype t, void *ws, size_t ws_bytes, void *stream) {
    if (any_null(q, dyq, dq) || (Hk > 0 && any_null(k, dyk, dk)) || (R > 0 && freq == nullptr)) return LA_ERR_NULL;
    const int st = qk_sizes(B, N, H, Hk, D, R, flags, t);
    if (st != LA_OK) return st;
    if (!(eps >= 0.0f) || !isfinite(eps) || ldq < H * D || (Hk > 0 && ldk < Hk * D) || (Hk == 0 && dwk != nullptr)) return LA_ERR_SHAPE;
    if (any_misaligned(q, k, wq, wk, freq, pos, lengths, dyq, dyk, dq, dk, dwq, dwk, ws)) return LA_ERR_ALIGN;
    la::QkArgs a = qk_args(B, N, H, Hk, D, R, flags, eps);
    const bool sums = dwq != nullptr || dwk != nullptr;
    const size_t need = sums ? qk_bytes(a) : 0;
    if (need > 0 && (ws == nullptr || ws_bytes < need)) return LA_ERR_WORKSPACE;
    const size_t T = (size_t)B * N, w = (size_t)D * 4, nq = span(T, H * D, H * D, t), nk = Hk > 0 ? span(T, Hk * D, Hk * D, t) : 0;
    const Span outs[] = {{dq, nq}, {dk, nk}, {dwq, span_of(dwq, w)}, {dwk, span_of(dwk, w)}, {ws, need}};
    const Span ins[] = {{q, span(T, ldq, H * D, t)}, {k, Hk > 0 ? span(T, ldk, Hk * D, t) : 0}, {dyq, nq}, {dyk, nk}, {wq, span_of(wq, w)},
                        {wk, span_of(wk, w)}, {freq, span_of(freq, (size_t)R * 2)}, {pos, span_of(pos, T * 4)}, {lengths, span_of(lengths, (size_t)B * 4)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    a.q = q, a.k = k, a.dyq = dyq, a.dyk = dyk, a.wq = wq, a.wk = wk, a.freq = freq, a.pos = pos, a.lengths = lengths, a.yq = dq, a.yk = dk;
    a.ldq = ldq, a.ldk = ldk, a.part = sums ? static_cast<float *>(ws) : nullptr;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int launched = hip_status(la::launch_qk_bwd(a, t, s));
    if (launched != LA_OK || !sums) return launched;
    return hip_status(la::launch_sum_rows(a.part, la::qk_groups(a), {{dwq, dwk, nullptr}, {D, D, 0}}, s));
}

size_t la_delta_fwd_workspace(int B, int N, int H, int Hk, int D, int M, la_dtype t, int flags) {
    if (delta_sizes(B, N, H, Hk, D, M, t, flags) != LA_OK) return 0;
    return Delta(B, N, H, Hk, D, M, 1.0f, t).fwd_bytes((flags & LA_DELTA_KEEP) != 0);
}

int la_delta_fwd(const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, const float *g, const float *beta, const float *h0,
                 const int *lengths, void *o, float *h1, int B, int N, int H, int Hk, int D, int M, float scale, int flags, la_dtype t,
                 void *ws, size_t ws_bytes, void *stream) {
    if (any_null(q, k, v, beta, o)) return LA_ERR_NULL;
    const int st = delta_sizes(B, N, H, Hk, D, M, t, flags);
    if (st != LA_OK) return st;
    if (!isfinite(scale) || bad_apart(ldq, Hk * D) || bad_apart(ldk, Hk * D) || bad_apart(ldv, H * M)) return LA_ERR_SHAPE;
    if (any_misaligned(q, k, v, g, beta, h0, lengths, o, h1, ws) || (ldq | ldk | ldv) % 8 != 0) return LA_ERR_ALIGN;
    Delta d(B, N, H, Hk, D, M, scale, t);
    const bool keep = (flags & LA_DELTA_KEEP) != 0;
    const size_t need = d.fwd_bytes(keep);
    if (ws == nullptr || ws_bytes < need) return LA_ERR_WORKSPACE;
    const size_t T = (size_t)B * N, per = T * H * 4, states = (size_t)B * H * D * M * 4;
    const Span outs[] = {{o, span(T, H * M, H * M, t)}, {h1, span_of(h1, states)}, {ws, need}};
    const Span ins[] = {{q, span(T, ldq, Hk * D, t)}, {k, span(T, ldk, Hk * D, t)}, {v, span(T, ldv, H * M, t)}, {g, span_of(g, per)}, {beta, per},
                        {h0, span_of(h0, states)}, {lengths, span_of(lengths, (size_t)B * 4)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::DeltaArgs &a = d.a;
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.h0 = h0, a.lengths = lengths, a.o = o, a.h1 = h1;
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    Carver cv{static_cast<char *>(ws), 0};
    d.carve_fwd(cv, keep);
    return hip_status(la::launch_delta_fwd(a, t, static_cast<hipStream_t>(stream)));
}

size_t la_delta_bwd_workspace(int B, int N, int H, int Hk, int D, int M, la_dtype t, int flags) {
    if (delta_sizes(B, N, H, Hk, D, M, t, flags) != LA_OK) return 0;
    return Delta(B, N, H, Hk, D, M, 1.0f, t).bwd_bytes((flags & LA_DELTA_KEEP) != 0);
}

int la_delta_bwd(const void *q, int ldq, const void *k, int ldk, const void *v, int ldv, const float *g, const float *beta, const float *h0,
                 const int *lengths, const void *fwd_ws, const void *dO, const float *dh1, void *dq, void *dk, void *dv, float *dg,
                 float *dbeta, float *dh0, int B, int N, int H, int Hk, int D, int M, float scale, int flags, la_dtype t, void *ws,
                 size_t ws_bytes, void *stream) {
    if (any_null(q, k, v, beta, dO, dq, dk, dv, dbeta) || (g == nullptr) != (dg == nullptr)) return LA_ERR_NULL;
    const int st = delta_sizes(B, N, H, Hk, D, M, t, flags);
    if (st != LA_OK) return st;
    if (!isfinite(scale) || bad_apart(ldq, Hk * D) || bad_apart(ldk, Hk * D) || bad_apart(ldv, H * M) || ((flags & LA_DELTA_KEEP) != 0) != (fwd_ws != nullptr)) return LA_ERR_SHAPE;
    if (any_misaligned(q, k, v, g, beta, h0, lengths, fwd_ws, dO, dh1, dq, dk, dv, dg, dbeta, dh0, ws) || (ldq | ldk | ldv) % 8 != 0) return LA_ERR_ALIGN;
    Delta d(B, N, H, Hk, D, M, scale, t);
    const bool given = fwd_ws != nullptr;
    const size_t need = d.bwd_bytes(given);
    if (ws == nullptr || ws_bytes < need) return LA_ERR_WORKSPACE;
    const size_t T = (size_t)B * N, per = T * H * 4, states = (size_t)B * H * D * M * 4, nk = span(T, Hk * D, Hk * D, t), nv = span(T, H * M, H * M, t);
    const Span outs[] = {{dq, nk}, {dk, nk}, {dv, nv}, {dg, span_of(dg, per)}, {dbeta, per}, {dh0, span_of(dh0, states)}, {ws, need}};
    const Span ins[] = {{q, span(T, ldq, Hk * D, t)}, {k, span(T, ldk, Hk * D, t)}, {v, span(T, ldv, H * M, t)}, {g, span_of(g, per)}, {beta, per},
                        {h0, span_of(h0, states)}, {lengths, span_of(lengths, (size_t)B * 4)}, {fwd_ws, given ? d.fwd_bytes(true) : 0}, {dO, nv},
                        {dh1, span_of(dh1, states)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::DeltaArgs &a = d.a;
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.h0 = h0, a.lengths = lengths;
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    Carver cv{static_cast<char *>(ws), 0};
    a.write = static_cast<float *>(cv.take(d.rows)), a.dstate = static_cast<float *>(cv.take(d.state));
    a.piece_dstate = static_cast<float *>(cv.take(d.pieces));
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (given) {
        Carver kept{static_cast<char *>(const_cast<void *>(fwd_ws)), 0};     // read only
        d.carve_fwd(kept, true);
    } else {
        d.carve_fwd(cv, true);
        const int formed = hip_status(la::launch_delta_fwd(a, t, s));
        if (formed != LA_OK) return formed;
    }
    a.dO = dO, a.dh1 = dh1, a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.dh0 = dh0;
    return hip_status(la::launch_delta_bwd(a, t, s));
}

int la_delta_step(const void *q, const void *k, const void *v, const float *g, const float *beta, float *h, void *o, int B, int H, int Hk,
                  int D, int M, float scale, la_dtype t, void *stream) {
    if (any_null(q, k, v, beta, h, o)) return LA_ERR_NULL;
    const int st = delta_sizes(B, 1, H, Hk, D, M, t, 0);
    if (st != LA_OK) return st;
    if (!isfinite(scale)) return LA_ERR_SHAPE;
    if (any_misaligned(q, k, v, g, beta, h, o)) return LA_ERR_ALIGN;
    const size_t e = esize_of(t), per = (size_t)B * H * 4, states = (size_t)B * H * D * M * 4;
    const Span outs[] = {{h, states}, {o, (size_t)B * H * M * e}};
    const Span ins[] = {{q, (size_t)B * Hk * D * e}, {k, (size_t)B * Hk * D * e}, {v, (size_t)B * H * M * e}, {g, span_of(g, per)}, {beta, per}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::DeltaArgs a{};
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.o = o;
    a.B = B, a.N = 1, a.H = H, a.Hk = Hk, a.D = D, a.M = M, a.scale = scale;
    return hip_status(la::launch_delta_step(a, h, t, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
