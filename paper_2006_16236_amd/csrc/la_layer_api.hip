// The C ABI of the operators around the attention: argument checks, workspace carving and launches.
#include <math.h>

#include "la_checks.h"
#include "la_layer.h"

namespace {
using namespace la_check;

int esize_of(la_dtype t) { return t == LA_BF16 ? 2 : 4; }
bool known(la_dtype t) { return t == LA_F32 || t == LA_BF16; }
// bytes from the first element of `rows` strided rows to behind the last one's `width` elements
size_t span(size_t rows, size_t ld, size_t width, la_dtype t) { return ((rows - 1) * ld + width) * esize_of(t); }
size_t span_of(const void *p, size_t bytes) { return p == nullptr ? 0 : bytes; }
template <typename... Ps> bool any_misaligned(Ps... p) { return (misaligned(p) || ...); }
template <typename... Ps> bool any_null(Ps... p) { return ((p == nullptr) || ...); }

// Tokens are counted in int, a run, a tile or two tiles ahead of the last one, and channels rounded up to a piece.
constexpr int kMostInt = 1 << 30;

// ---- layer norm ---------------------------------------------------------------------------------
constexpr int kMaxNorm = 16384;

int norm_sizes(int rows, int E, la_dtype t) {
    if (!known(t)) return LA_ERR_UNSUPPORTED;
    if (rows < 1 || E < 1) return LA_ERR_SHAPE;
    if (E > kMaxNorm) return LA_ERR_UNSUPPORTED;
    return LA_OK;
}
size_t norm_bytes(int rows, int E, la_dtype t) { return align256((size_t)la::norm_groups(rows, E, t) * 2 * E * sizeof(float)); }

// ---- convolution --------------------------------------------------------------------------------
int conv_sizes(int B, int N, int E, int W, la_dtype t) {
    if (!known(t)) return LA_ERR_UNSUPPORTED;
    if (W < 2 || W > 4) return LA_ERR_UNSUPPORTED;
    if (B < 1 || N < 1 || E < 1 || N > kMostInt || E > kMostInt) return LA_ERR_SHAPE;
    if ((double)B * N * E >= 68719476736.0) return LA_ERR_SHAPE;                                    // 2^36
    if ((double)B * ((double)(N - 1) / 8 + 1) * (E / 4 + 1.0) >= 2147483648.0) return LA_ERR_SHAPE;  // threads of a launch
    return LA_OK;
}
size_t conv_bytes(int B, int N, int E, int W) {
    la::ConvArgs a{};
    a.B = B, a.N = N, a.E = E, a.W = W;
    return align256((size_t)la::conv_plan_bwd(a) * E * (W + 1) * sizeof(float));
}

// ---- scan ---------------------------------------------------------------------------------------
int scan_sizes(int B, int N, int E, int G, int S, la_dtype t, int flags) {
    if (!known(t) || !(S == 8 || S == 16 || S == 32) || (flags & ~(LA_SCAN_SOFTPLUS | LA_SCAN_KEEP)) != 0) return LA_ERR_UNSUPPORTED;
    if (B < 1 || N < 1 || E < 1 || G < 1 || E % G != 0 || N > kMostInt) return LA_ERR_SHAPE;
    if ((double)B * N * E >= 68719476736.0 || (double)B * E >= 268435456.0) return LA_ERR_SHAPE;     // 2^36, 2^28
    if ((double)B * la::scan_blocks(E, G) >= 8388608.0) return LA_ERR_SHAPE;                         // 2^23 workgroups
    if ((double)B * N * G * S >= 68719476736.0 || (double)G * S >= 2147483648.0) return LA_ERR_SHAPE;
    return LA_OK;
}
// a scan's sizes, and the parts of its workspace.  Each pass has its own cut; what the forward keeps does not depend on it.
struct Scan {
    la::ScanArgs a{};
    size_t states, keep, part_bc;
    Scan(int B, int N, int E, int G, int S) {
        a.B = B, a.N = N, a.E = E, a.G = G, a.S = S;
        la::scan_cut(a, false);
        states = (size_t)B * E * S * sizeof(float);
        keep = align256(states * a.tiles);
        part_bc = align256((size_t)la::scan_blocks(E, G) * B * N * 2 * S * sizeof(float));
    }
    size_t pieces_bytes() const {
        if (a.pieces < 2) return 0;
        return align256(states * a.pieces) + align256((size_t)a.B * a.pieces * a.E * sizeof(float));
    }
    size_t part_bytes() const { return align256((size_t)a.B * a.pieces * a.E * (a.S + 2) * sizeof(float)); }
    void carve_pieces(Carver &cv) {
        if (a.pieces < 2) return;
        a.piece_h = static_cast<float *>(cv.take(states * a.pieces));
        a.piece_d = static_cast<float *>(cv.take((size_t)a.B * a.pieces * a.E * sizeof(float)));
    }
    // the kept states come first: the backward finds them at the workspace's start
    size_t fwd_bytes(int flags) const { return (flags & LA_SCAN_KEEP ? keep : 0) + pieces_bytes(); }
    // without the forward's states these are formed here, by a forward whose pieces' states share the backward's room
    size_t bwd_bytes(int flags) const {
        Scan back = *this;
        la::scan_cut(back.a, true);
        const size_t mine = back.pieces_bytes(), rebuilt = flags & LA_SCAN_KEEP ? 0 : pieces_bytes();
        return (flags & LA_SCAN_KEEP ? 0 : keep) + (mine > rebuilt ? mine : rebuilt) + part_bc + back.part_bytes();
    }
};
bool bad_rows(int ld, int width) { return ld < width; }
}  // namespace

extern "C" {

int la_norm_fwd(const void *x, const void *r, const float *gamma, const float *beta, void *y, void *s, float *mean, float *rstd,
                int rows, int E, float eps, la_dtype t, void *stream) {
    if (any_null(x, y)) return LA_ERR_NULL;
    if (s != nullptr && r == nullptr) return LA_ERR_NULL;
    const int st = norm_sizes(rows, E, t);
    if (st != LA_OK) return st;
    if (!(eps >= 0.0f) || !isfinite(eps)) return LA_ERR_SHAPE;
    if (any_misaligned(x, r, gamma, beta, y, s, mean, rstd)) return LA_ERR_ALIGN;
    const size_t n = (size_t)rows * E * esize_of(t), col = (size_t)E * 4, per = (size_t)rows * 4;
    const Span outs[] = {{y, n}, {s, span_of(s, n)}, {mean, span_of(mean, per)}, {rstd, span_of(rstd, per)}};
    const Span ins[] = {{x, n}, {r, span_of(r, n)}, {gamma, span_of(gamma, col)}, {beta, span_of(beta, col)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::NormArgs a{};
    a.x = x, a.r = r, a.gamma = gamma, a.beta = beta, a.y = y, a.s = s, a.mean = mean, a.rstd = rstd;
    a.rows = rows, a.E = E, a.eps = eps;
    return hip_status(la::launch_norm_fwd(a, t, static_cast<hipStream_t>(stream)));
}

size_t la_norm_bwd_workspace(int rows, int E, la_dtype t) { return norm_sizes(rows, E, t) == LA_OK ? norm_bytes(rows, E, t) : 0; }

int la_norm_bwd(const void *s, const float *gamma, const float *mean, const float *rstd, const void *dy, const void *ds, void *dx,
                float *dgamma, float *dbeta, int rows, int E, la_dtype t, void *ws, size_t ws_bytes, void *stream) {
    if (any_null(s, mean, rstd, dy, dx)) return LA_ERR_NULL;
    const int st = norm_sizes(rows, E, t);
    if (st != LA_OK) return st;
    if (any_misaligned(s, gamma, mean, rstd, dy, ds, dx, dgamma, dbeta, ws)) return LA_ERR_ALIGN;
    const bool sums = dgamma != nullptr || dbeta != nullptr;
    const size_t need = sums ? norm_bytes(rows, E, t) : 0;
    if (need > 0 && (ws == nullptr || ws_bytes < need)) return LA_ERR_WORKSPACE;
    const size_t n = (size_t)rows * E * esize_of(t), col = (size_t)E * 4, per = (size_t)rows * 4;
    const Span outs[] = {{dx, n}, {dgamma, span_of(dgamma, col)}, {dbeta, span_of(dbeta, col)}, {ws, need}};
    const Span ins[] = {{s, n}, {dy, n}, {ds, span_of(ds, n)}, {gamma, span_of(gamma, col)}, {mean, per}, {rstd, per}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::NormArgs a{};
    a.x = s, a.r = ds, a.dy = dy, a.gamma = gamma, a.mean_in = mean, a.rstd_in = rstd, a.y = dx;
    a.part = sums ? static_cast<float *>(ws) : nullptr, a.dgamma = dgamma, a.dbeta = dbeta;
    a.rows = rows, a.E = E;
    hipStream_t q = static_cast<hipStream_t>(stream);
    const int launched = hip_status(la::launch_norm_bwd(a, t, q));
    const int groups = la::norm_groups(rows, E, t);
    if (launched != LA_OK || !sums || groups == 1) return launched;
    return hip_status(la::launch_sum_rows(a.part, groups, {{dgamma, dbeta, nullptr}, {E, E, 0}}, q));
}

int la_conv_fwd(const void *x, int ldx, const float *w, const float *bias, const void *x0, const int *lengths, void *y, void *x1,
                int B, int N, int E, int W, int silu, la_dtype t, void *stream) {
    if (any_null(x, w, y)) return LA_ERR_NULL;
    const int st = conv_sizes(B, N, E, W, t);
    if (st != LA_OK) return st;
    if (bad_rows(ldx, E)) return LA_ERR_SHAPE;
    if (any_misaligned(x, w, bias, x0, lengths, y, x1)) return LA_ERR_ALIGN;
    const size_t rows = (size_t)B * N, e = esize_of(t), state = (size_t)B * (W - 1) * E * e;
    const Span outs[] = {{y, rows * E * e}, {x1, span_of(x1, state)}};
    const Span ins[] = {{x, span(rows, ldx, E, t)}, {w, (size_t)E * W * 4}, {bias, span_of(bias, (size_t)E * 4)},
                        {x0, span_of(x0, state)}, {lengths, span_of(lengths, (size_t)B * 4)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::ConvArgs a{};
    a.x = x, a.x0 = x0, a.w = w, a.bias = bias, a.lengths = lengths, a.y = y, a.x1 = x1, a.ldx = ldx;
    a.B = B, a.N = N, a.E = E, a.W = W, a.silu = silu != 0;
    return hip_status(la::launch_conv_fwd(a, t, static_cast<hipStream_t>(stream)));
}

size_t la_conv_bwd_workspace(int B, int N, int E, int W, la_dtype t) {
    return conv_sizes(B, N, E, W, t) == LA_OK ? conv_bytes(B, N, E, W) : 0;
}

int la_conv_bwd(const void *x, int ldx, const float *w, const float *bias, const void *x0, const int *lengths, const void *dy,
                const void *dx1, void *dx, float *dw, float *db, void *dx0, int B, int N, int E, int W, int silu, la_dtype t,
                void *ws, size_t ws_bytes, void *stream) {
    if (any_null(x, w, dy, dx)) return LA_ERR_NULL;
    const int st = conv_sizes(B, N, E, W, t);
    if (st != LA_OK) return st;
    if (bad_rows(ldx, E)) return LA_ERR_SHAPE;
    if (any_misaligned(x, w, bias, x0, lengths, dy, dx1, dx, dw, db, dx0, ws)) return LA_ERR_ALIGN;
    const bool sums = dw != nullptr || db != nullptr;
    const size_t need = sums ? conv_bytes(B, N, E, W) : 0;
    if (need > 0 && (ws == nullptr || ws_bytes < need)) return LA_ERR_WORKSPACE;
    const size_t rows = (size_t)B * N, e = esize_of(t), state = (size_t)B * (W - 1) * E * e, taps = (size_t)E * W * 4, col = (size_t)E * 4;
    const Span outs[] = {{dx, rows * E * e}, {dw, span_of(dw, taps)}, {db, span_of(db, col)}, {dx0, span_of(dx0, state)}, {ws, need}};
    const Span ins[] = {{x, span(rows, ldx, E, t)}, {w, taps}, {bias, span_of(bias, col)}, {x0, span_of(x0, state)},
                        {lengths, span_of(lengths, (size_t)B * 4)}, {dy, rows * E * e}, {dx1, span_of(dx1, state)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::ConvArgs a{};
    a.x = x, a.x0 = x0, a.w = w, a.bias = bias, a.lengths = lengths, a.dy = dy, a.dx1 = dx1, a.dx = dx, a.dx0 = dx0, a.ldx = ldx;
    a.part = sums ? static_cast<float *>(ws) : nullptr;
    a.B = B, a.N = N, a.E = E, a.W = W, a.silu = silu != 0;
    const long parts = la::conv_plan_bwd(a);
    hipStream_t q = static_cast<hipStream_t>(stream);
    const int launched = hip_status(la::launch_conv_bwd(a, t, q));
    if (launched != LA_OK || !sums) return launched;
    return hip_status(la::launch_sum_rows(a.part, parts, {{dw, db, nullptr}, {(long)E * W, E, 0}}, q));
}

int la_conv_step(const void *x, const float *w, const float *bias, void *state, void *y, int B, int E, int W, int silu, la_dtype t,
                 void *stream) {
    if (any_null(x, w, state, y)) return LA_ERR_NULL;
    const int st = conv_sizes(B, 1, E, W, t);
    if (st != LA_OK) return st;
    if (any_misaligned(x, w, bias, state, y)) return LA_ERR_ALIGN;
    const size_t row = (size_t)B * E * esize_of(t);
    const Span outs[] = {{y, row}, {state, row * (W - 1)}};
    const Span ins[] = {{x, row}, {w, (size_t)E * W * 4}, {bias, span_of(bias, (size_t)E * 4)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    return hip_status(la::launch_conv_step(x, w, bias, state, y, B, E, W, silu != 0, t, static_cast<hipStream_t>(stream)));
}

size_t la_scan_fwd_workspace(int B, int N, int E, int G, int S, la_dtype t, int flags) {
    return scan_sizes(B, N, E, G, S, t, flags) == LA_OK ? Scan(B, N, E, G, S).fwd_bytes(flags) : 0;
}

int la_scan_fwd(const void *x, int ldx, const void *dt, int lddt, const void *z, int ldz, const void *Bt, int ldb, const void *Ct,
                int ldc, const float *A, const float *D, const float *dt_bias, const float *h0, const int *lengths, void *y, float *h1,
                int B, int N, int E, int G, int S, int flags, la_dtype t, void *ws, size_t ws_bytes, void *stream) {
    if (any_null(x, dt, Bt, Ct, A, y)) return LA_ERR_NULL;
    const int st = scan_sizes(B, N, E, G, S, t, flags);
    if (st != LA_OK) return st;
    if (bad_rows(ldx, E) || bad_rows(lddt, E) || (z != nullptr && bad_rows(ldz, E)) || bad_rows(ldb, G * S) || bad_rows(ldc, G * S))
        return LA_ERR_SHAPE;
    if (any_misaligned(x, dt, z, Bt, Ct, A, D, dt_bias, h0, lengths, y, h1, ws))
        return LA_ERR_ALIGN;
    Scan k(B, N, E, G, S);
    const size_t need = k.fwd_bytes(flags);
    if (need > 0 && (ws == nullptr || ws_bytes < need)) return LA_ERR_WORKSPACE;
    const size_t rows = (size_t)B * N, col = (size_t)E * 4, states = (size_t)B * E * S * 4;
    const Span outs[] = {{y, rows * E * esize_of(t)}, {h1, span_of(h1, states)}, {ws, need}};
    const Span ins[] = {{x, span(rows, ldx, E, t)}, {dt, span(rows, lddt, E, t)}, {z, span_of(z, span(rows, ldz, E, t))},
                        {Bt, span(rows, ldb, (size_t)G * S, t)}, {Ct, span(rows, ldc, (size_t)G * S, t)}, {A, col * S},
                        {D, span_of(D, col)}, {dt_bias, span_of(dt_bias, col)}, {h0, span_of(h0, states)},
                        {lengths, span_of(lengths, (size_t)B * 4)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::ScanArgs &a = k.a;
    a.x = x, a.dt = dt, a.z = z, a.Bt = Bt, a.Ct = Ct, a.A = A, a.D = D, a.bias = dt_bias, a.h0 = h0, a.lengths = lengths;
    a.y = y, a.h1 = h1, a.ldx = ldx, a.lddt = lddt, a.ldz = ldz, a.ldb = ldb, a.ldc = ldc;
    a.softplus = (flags & LA_SCAN_SOFTPLUS) != 0;
    Carver cv{static_cast<char *>(ws), 0};
    if (flags & LA_SCAN_KEEP) a.keep = static_cast<float *>(cv.take(k.keep));
    k.carve_pieces(cv);
    return hip_status(la::launch_scan_fwd(a, t, static_cast<hipStream_t>(stream)));
}

size_t la_scan_bwd_workspace(int B, int N, int E, int G, int S, la_dtype t, int flags) {
    return scan_sizes(B, N, E, G, S, t, flags) == LA_OK ? Scan(B, N, E, G, S).bwd_bytes(flags) : 0;
}

int la_scan_bwd(const void *x, int ldx, const void *dt, int lddt, const void *z, int ldz, const void *Bt, int ldb, const void *Ct,
                int ldc, const float *A, const float *D, const float *dt_bias, const float *h0, const int *lengths, const void *fwd_ws,
                const void *dy, const float *dh1, void *dx, void *ddt, void *dz, void *dB, void *dC, float *dA, float *dD,
                float *ddt_bias, float *dh0, int B, int N, int E, int G, int S, int flags, la_dtype t, void *ws, size_t ws_bytes,
                void *stream) {
    if (any_null(x, dt, Bt, Ct, A, dy, dx, ddt, dB, dC, dA)) return LA_ERR_NULL;
    if ((z == nullptr) != (dz == nullptr)) return LA_ERR_NULL;
    const int st = scan_sizes(B, N, E, G, S, t, flags);
    if (st != LA_OK) return st;
    if (bad_rows(ldx, E) || bad_rows(lddt, E) || (z != nullptr && bad_rows(ldz, E)) || bad_rows(ldb, G * S) || bad_rows(ldc, G * S))
        return LA_ERR_SHAPE;
    if (any_misaligned(x, dt, z, Bt, Ct, A, D, dt_bias, h0, lengths, fwd_ws, dy, dh1, dx, ddt, dz, dB, dC, dA, dD, ddt_bias, dh0, ws))
        return LA_ERR_ALIGN;
    Scan k(B, N, E, G, S);
    const size_t need = k.bwd_bytes(fwd_ws != nullptr ? LA_SCAN_KEEP : 0);
    if (ws == nullptr || ws_bytes < need) return LA_ERR_WORKSPACE;
    const size_t rows = (size_t)B * N, big = rows * E * esize_of(t), bc = rows * G * S * esize_of(t), col = (size_t)E * 4;
    const size_t states = (size_t)B * E * S * 4;
    const Span outs[] = {{dx, big}, {ddt, big}, {dz, span_of(dz, big)}, {dB, bc}, {dC, bc}, {dA, col * S}, {dD, span_of(dD, col)},
                         {ddt_bias, span_of(ddt_bias, col)}, {dh0, span_of(dh0, states)}, {ws, need}};
    const Span ins[] = {{x, span(rows, ldx, E, t)}, {dt, span(rows, lddt, E, t)}, {z, span_of(z, span(rows, ldz, E, t))},
                        {Bt, span(rows, ldb, (size_t)G * S, t)}, {Ct, span(rows, ldc, (size_t)G * S, t)}, {A, col * S},
                        {D, span_of(D, col)}, {dt_bias, span_of(dt_bias, col)}, {h0, span_of(h0, states)},
                        {lengths, span_of(lengths, (size_t)B * 4)}, {fwd_ws, span_of(fwd_ws, k.keep)}, {dy, big},
                        {dh1, span_of(dh1, states)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::ScanArgs &a = k.a;
    a.x = x, a.dt = dt, a.z = z, a.Bt = Bt, a.Ct = Ct, a.A = A, a.D = D, a.bias = dt_bias, a.h0 = h0, a.lengths = lengths;
    a.dy = dy, a.dh1 = dh1, a.dx = dx, a.ddt = ddt, a.dz = dz, a.dB = dB, a.dC = dC, a.dh0 = dh0;
    a.ldx = ldx, a.lddt = lddt, a.ldz = ldz, a.ldb = ldb, a.ldc = ldc;
    a.softplus = (flags & LA_SCAN_SOFTPLUS) != 0;
    Carver cv{static_cast<char *>(ws), 0};
    hipStream_t q = static_cast<hipStream_t>(stream);
    if (fwd_ws != nullptr) {
        a.keep = const_cast<float *>(static_cast<const float *>(fwd_ws));
    } else {
        a.keep = static_cast<float *>(cv.take(k.keep));
        Carver shared = cv;
        k.carve_pieces(shared);
        const int done = hip_status(la::launch_scan_fwd(a, t, q));                 // no outputs but the states before each tile
        if (done != LA_OK) return done;
    }
    const size_t forward = fwd_ws != nullptr ? 0 : k.pieces_bytes();
    la::scan_cut(a, true);
    const size_t mine = k.pieces_bytes();
    Carver pieces = cv;
    k.carve_pieces(pieces);
    cv.off += mine > forward ? mine : forward;
    a.part_bc = static_cast<float *>(cv.take(k.part_bc));
    a.part = static_cast<float *>(cv.take(k.part_bytes()));
    const int done = hip_status(la::launch_scan_bwd(a, t, q));
    if (done != LA_OK) return done;
    return hip_status(la::launch_sum_rows(a.part, (long)B * a.pieces, {{dA, dD, ddt_bias}, {(long)E * S, E, E}}, q));
}

int la_scan_step(const void *x, const void *dt, const void *z, const void *Bt, const void *Ct, const float *A, const float *D,
                 const float *dt_bias, float *h, void *y, int B, int E, int G, int S, int flags, la_dtype t, void *stream) {
    if (any_null(x, dt, Bt, Ct, A, h, y)) return LA_ERR_NULL;
    const int st = scan_sizes(B, 1, E, G, S, t, flags);
    if (st != LA_OK) return st;
    if (flags & LA_SCAN_KEEP) return LA_ERR_UNSUPPORTED;
    if ((double)B * (E * (S / 4.0) + 256) >= 4294967296.0) return LA_ERR_SHAPE;
    if (any_misaligned(x, dt, z, Bt, Ct, A, D, dt_bias, h, y)) return LA_ERR_ALIGN;
    const size_t row = (size_t)B * E * esize_of(t), bc = (size_t)B * G * S * esize_of(t), col = (size_t)E * 4;
    const Span outs[] = {{y, row}, {h, (size_t)B * E * S * 4}};
    const Span ins[] = {{x, row}, {dt, row}, {z, span_of(z, row)}, {Bt, bc}, {Ct, bc}, {A, col * S}, {D, span_of(D, col)},
                        {dt_bias, span_of(dt_bias, col)}};
    if (aliased(outs, ins)) return LA_ERR_ALIAS;
    la::ScanArgs a{};
    a.x = x, a.dt = dt, a.z = z, a.Bt = Bt, a.Ct = Ct, a.A = A, a.D = D, a.bias = dt_bias, a.y = y;
    a.B = B, a.N = 1, a.E = E, a.G = G, a.S = S, a.softplus = (flags & LA_SCAN_SOFTPLUS) != 0;
    return hip_status(la::launch_scan_step(a, h, t, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
