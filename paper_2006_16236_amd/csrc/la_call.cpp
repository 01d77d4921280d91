// The accepting path of the binding's calls in native code: checks the tensors of a call and hands their
// pointers to the C ABI.  A decode step is a 5 us kernel; checking six tensors and marshalling thirteen
// arguments in Python took the host 9.
//
// Every function answers None when it does not take the call (an argument that is not a plain dense
// device tensor of the expected sizes, an option it does not know); the caller then goes through its own
// checks, which name what is wrong.  Nothing is kept between calls.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include <initializer_list>

namespace {

// addresses of the library's entry points, set once by bind()
typedef int (*step_fn)(const void *, const void *, const void *, float *, float *, void *, int, int, int, int, float, int, void *);
typedef int (*fwd_fn)(const void *, const void *, const void *, void *, float *, int, int, int, int, int, float, int, void *,
                      size_t, void *);
typedef int (*bwd_fn)(const void *, const void *, const void *, const void *, const float *, const void *, const void *, void *,
                      void *, void *, int, int, int, int, int, float, int, void *, size_t, void *);
typedef size_t (*ws_fn)(int, int, int, int, int, int);
step_fn g_step = nullptr;
// causal, causal token-major, non-causal, non-causal token-major; workspaces: causal, non-causal
fwd_fn g_fwd[4] = {};
bwd_fn g_bwd[4] = {};
ws_fn g_fwd_ws[2] = {}, g_bwd_ws[2] = {};

// a plain dense tensor on a device: no subclass, no wrapper of a transform, no mode's stand-in
const at::Tensor *plain(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    static const c10::DispatchKeySet wrappers{c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                              c10::DispatchKey::Functionalize, c10::DispatchKey::Python};
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.key_set().has_any(wrappers)) return nullptr;
    return t.is_contiguous() ? &t : nullptr;
}
// ... of these sizes, element type and device
const at::Tensor *like(PyObject *o, at::IntArrayRef sizes, at::ScalarType dt, const at::Device &dev) {
    const at::Tensor *t = plain(o);
    return t != nullptr && t->sizes() == sizes && t->scalar_type() == dt && t->device() == dev ? t : nullptr;
}
// element-type code of a call, -1: not taken here
int type_code(at::ScalarType dt, PyObject *features) {
    const int base = dt == at::kFloat ? 0 : dt == at::kBFloat16 ? 1 : -1;
    if (base < 0) return -1;
    return features == Py_False ? base : features == Py_True ? base + 2 : -1;
}
void *stream() { return c10::hip::getCurrentHIPStream().stream(); }
bool fits(const at::Tensor &t) {       // sizes the C ABI takes as int
    for (const int64_t n : t.sizes())
        if (n > 0x7fffffff) return false;
    return true;
}
PyObject *not_taken() { Py_RETURN_NONE; }

// step(q, k, v, S, z, out, eps, features) -> status
PyObject *py_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 8 || g_step == nullptr) return not_taken();
    const double eps = PyFloat_AsDouble(a[6]);
    if (eps == -1.0 && PyErr_Occurred()) return nullptr;
    int st;
    try {
        const at::Tensor *q = plain(a[0]), *v = plain(a[2]);
        if (q == nullptr || v == nullptr || q->dim() != 3 || v->dim() != 3 || !fits(*q) || !fits(*v)) return not_taken();
        const int64_t B = q->size(0), H = q->size(1), D = q->size(2), M = v->size(2);
        const at::ScalarType dt = q->scalar_type();
        const at::Device dev = q->device();
        const int code = type_code(dt, a[7]);
        const at::Tensor *k = like(a[1], q->sizes(), dt, dev), *out = like(a[5], v->sizes(), dt, dev);
        const at::Tensor *S = like(a[3], {B, H, D, M}, at::kFloat, dev), *z = like(a[4], {B, H, D}, at::kFloat, dev);
        if (code < 0 || k == nullptr || out == nullptr || S == nullptr || z == nullptr || v->size(0) != B || v->size(1) != H ||
            v->scalar_type() != dt || v->device() != dev)
            return not_taken();
        const void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr();
        float *pS = static_cast<float *>(S->data_ptr()), *pz = static_cast<float *>(z->data_ptr());
        void *po = out->data_ptr(), *s = stream();
        Py_BEGIN_ALLOW_THREADS
        st = g_step(pq, pk, pv, pS, pz, po, (int)B, (int)H, (int)D, (int)M, (float)eps, code, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        return not_taken();
    }
    return PyLong_FromLong(st);
}

struct Sizes {
    int64_t B, H, N, D, M;
    at::ScalarType dt;
    at::Device dev = at::Device(at::kCPU);
    int code;
};
// Q, K, V of an N-sized call; kind & 1: token-major
bool inputs(int kind, PyObject *q, PyObject *k, PyObject *v, PyObject *features, Sizes &z, const at::Tensor *(&t)[3]) {
    t[0] = plain(q), t[2] = plain(v);
    if (t[0] == nullptr || t[2] == nullptr || t[0]->dim() != 4 || t[2]->dim() != 4 || !fits(*t[0]) || !fits(*t[2])) return false;
    z.dt = t[0]->scalar_type(), z.dev = t[0]->device();
    z.code = type_code(z.dt, features);
    z.B = t[0]->size(0), z.H = t[0]->size(kind & 1 ? 2 : 1), z.N = t[0]->size(kind & 1 ? 1 : 2), z.D = t[0]->size(3), z.M = t[2]->size(3);
    t[1] = like(k, t[0]->sizes(), z.dt, z.dev);
    return z.code >= 0 && t[1] != nullptr && t[2]->scalar_type() == z.dt && t[2]->device() == z.dev &&
           t[2]->sizes().slice(0, 3) == t[0]->sizes().slice(0, 3);
}
// a workspace: the caller's (any dense tensor on the device), or a new one
bool workspace(PyObject *o, size_t need, const Sizes &z, at::Tensor &ws) {
    if (o == Py_None) {
        ws = at::empty({(int64_t)(need > 16 ? need : 16)}, at::TensorOptions().dtype(at::kByte).device(z.dev));
        return true;
    }
    const at::Tensor *t = plain(o);
    if (t == nullptr || t->device() != z.dev) return false;
    ws = *t;
    return true;
}
PyObject *answer(int st, PyObject *given, const at::Tensor &ws) {
    if (st != 0) return PyLong_FromLong(st);
    if (given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    return THPVariable_Wrap(ws);
}

// fwd(kind, Q, K, V, O, den | None, ws | None, eps, features) -> the workspace, or the status of a failed call
PyObject *py_fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) return not_taken();
    const long kind = PyLong_AsLong(a[0]);
    const double eps = PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) return nullptr;
    if (kind < 0 || kind > 3 || g_fwd[kind] == nullptr) return not_taken();
    try {
        Sizes z;
        const at::Tensor *in[3], *den = nullptr;
        if (!inputs((int)kind, a[1], a[2], a[3], a[8], z, in)) return not_taken();
        const at::Tensor *O = like(a[4], in[2]->sizes(), z.dt, z.dev);
        if (a[5] != Py_None) den = like(a[5], {z.B, z.H, z.N}, at::kFloat, z.dev);
        if (O == nullptr || (a[5] != Py_None && den == nullptr)) return not_taken();
        at::Tensor ws;
        if (!workspace(a[6], g_fwd_ws[kind >> 1]((int)z.B, (int)z.H, (int)z.N, (int)z.D, (int)z.M, z.code), z, ws)) return not_taken();
        const void *q = in[0]->data_ptr(), *k = in[1]->data_ptr(), *v = in[2]->data_ptr();
        void *o = O->data_ptr(), *w = ws.data_ptr(), *s = stream();
        float *d = den != nullptr ? static_cast<float *>(den->data_ptr()) : nullptr;
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = g_fwd[kind](q, k, v, o, d, (int)z.B, (int)z.H, (int)z.N, (int)z.D, (int)z.M, (float)eps, z.code, w, ws.nbytes(), s);
        Py_END_ALLOW_THREADS
        return answer(st, a[6], ws);
    } catch (...) {
        return not_taken();
    }
}

// bwd(kind, Q, K, V, O | None, den, dO, dQ, dK, dV, ws | None, fwd_ws, eps, features) -> as fwd
PyObject *py_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 14) return not_taken();
    const long kind = PyLong_AsLong(a[0]);
    const double eps = PyFloat_AsDouble(a[12]);
    if (PyErr_Occurred()) return nullptr;
    if (kind < 0 || kind > 3 || g_bwd[kind] == nullptr || a[5] == Py_None || a[11] == Py_None) return not_taken();
    try {
        Sizes z;
        const at::Tensor *in[3];
        if (!inputs((int)kind, a[1], a[2], a[3], a[13], z, in)) return not_taken();
        const at::IntArrayRef qk = in[0]->sizes(), vv = in[2]->sizes();
        const at::Tensor *den = like(a[5], {z.B, z.H, z.N}, at::kFloat, z.dev), *g = like(a[6], vv, z.dt, z.dev);
        const at::Tensor *dq = like(a[7], qk, z.dt, z.dev), *dk = like(a[8], qk, z.dt, z.dev), *dv = like(a[9], vv, z.dt, z.dev);
        const at::Tensor *fws = plain(a[11]);
        if (den == nullptr || g == nullptr || dq == nullptr || dk == nullptr || dv == nullptr || fws == nullptr || fws->device() != z.dev ||
            (a[4] != Py_None && like(a[4], vv, z.dt, z.dev) == nullptr) ||
            fws->nbytes() < g_fwd_ws[kind >> 1]((int)z.B, (int)z.H, (int)z.N, (int)z.D, (int)z.M, z.code))
            return not_taken();
        at::Tensor ws;
        if (!workspace(a[10], g_bwd_ws[kind >> 1]((int)z.B, (int)z.H, (int)z.N, (int)z.D, (int)z.M, z.code), z, ws)) return not_taken();
        const void *q = in[0]->data_ptr(), *k = in[1]->data_ptr(), *v = in[2]->data_ptr(), *gp = g->data_ptr(), *fp = fws->data_ptr();
        const void *o = a[4] != Py_None ? THPVariable_Unpack(a[4]).data_ptr() : nullptr;
        const float *d = static_cast<const float *>(den->data_ptr());
        void *pq = dq->data_ptr(), *pk = dk->data_ptr(), *pv = dv->data_ptr(), *w = ws.data_ptr(), *s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = g_bwd[kind](q, k, v, o, d, fp, gp, pq, pk, pv, (int)z.B, (int)z.H, (int)z.N, (int)z.D, (int)z.M, (float)eps, z.code, w,
                         ws.nbytes(), s);
        Py_END_ALLOW_THREADS
        return answer(st, a[10], ws);
    } catch (...) {
        return not_taken();
    }
}

// ---- the operators around the attention ----------------------------------------------------------
// The arguments of the functions of the same names in layer.py, in their order, without the stream.

struct Layer {                       // addresses of the library's entry points, set once by bind_layer()
    int (*norm_fwd)(const void *, const void *, const float *, const float *, void *, void *, float *, float *, int, int, float, int, void *);
    size_t (*norm_bwd_ws)(int, int, int);
    int (*norm_bwd)(const void *, const float *, const float *, const float *, const void *, const void *, void *, float *, float *, int,
                    int, int, void *, size_t, void *);
    int (*conv_fwd)(const void *, int, const float *, const float *, const void *, const int *, void *, void *, int, int, int, int, int,
                    int, void *);
    size_t (*conv_bwd_ws)(int, int, int, int, int);
    int (*conv_bwd)(const void *, int, const float *, const float *, const void *, const int *, const void *, const void *, void *, float *,
                    float *, void *, int, int, int, int, int, int, void *, size_t, void *);
    int (*conv_step)(const void *, const float *, const float *, void *, void *, int, int, int, int, int, void *);
    size_t (*scan_fwd_ws)(int, int, int, int, int, int, int);
    int (*scan_fwd)(const void *, int, const void *, int, const void *, int, const void *, int, const void *, int, const float *,
                    const float *, const float *, const float *, const int *, void *, float *, int, int, int, int, int, int, int, void *,
                    size_t, void *);
    size_t (*scan_bwd_ws)(int, int, int, int, int, int, int);
    int (*scan_bwd)(const void *, int, const void *, int, const void *, int, const void *, int, const void *, int, const float *,
                    const float *, const float *, const float *, const int *, const void *, const void *, const float *, void *, void *,
                    void *, void *, void *, float *, float *, float *, float *, int, int, int, int, int, int, int, void *, size_t, void *);
    int (*scan_step)(const void *, const void *, const void *, const void *, const void *, const float *, const float *, const float *,
                     float *, void *, int, int, int, int, int, int, void *);
} g_layer = {};

// Collects the pointers of a call's tensors; ok goes to false at the first one that is not as expected.
struct Taker {
    bool ok = true;
    at::ScalarType dt = at::kFloat;
    at::Device dev = at::Device(at::kCPU);
    int code = -1;
    // the tensor that says the call's type and device; launches go to the current device
    const at::Tensor *lead(PyObject *o, int64_t dim) {
        const at::Tensor *t = tensor(o);
        if (t == nullptr || t->dim() != dim || t->numel() == 0 || !fits(*t)) return fail();
        dt = t->scalar_type(), dev = t->device();
        code = dt == at::kFloat ? 0 : dt == at::kBFloat16 ? 1 : -1;
        if (code < 0 || dev.index() != c10::hip::current_device()) return fail();
        return t;
    }
    const at::Tensor *fail() {
        ok = false;
        return nullptr;
    }
    static const at::Tensor *tensor(PyObject *o) {
        if (!THPVariable_CheckExact(o)) return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        static const c10::DispatchKeySet wrappers{c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                                  c10::DispatchKey::Functionalize, c10::DispatchKey::Python};
        return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.key_set().has_any(wrappers) ? &t : nullptr;
    }
    // a dense tensor of the call's type (or fp32, int32); None where that is allowed
    void *dense(PyObject *o, at::IntArrayRef sizes, at::ScalarType type, bool optional = false) {
        if (!ok || (optional && o == Py_None)) return nullptr;
        const at::Tensor *t = tensor(o);
        if (t == nullptr || t->sizes() != sizes || t->scalar_type() != type || t->device() != dev || !t->is_contiguous()) return ok = false, nullptr;
        return t->data_ptr();
    }
    void *mine(PyObject *o, at::IntArrayRef sizes, bool optional = false) { return dense(o, sizes, dt, optional); }
    float *f32(PyObject *o, at::IntArrayRef sizes, bool optional = false) { return static_cast<float *>(dense(o, sizes, at::kFloat, optional)); }
    // rows [B, N, ..] of the call's type whose tokens lie at one distance, `ld`
    const void *rows(PyObject *o, at::IntArrayRef sizes, int &ld, bool optional = false) {
        ld = 0;
        if (!ok || (optional && o == Py_None)) return nullptr;
        const at::Tensor *t = tensor(o);
        if (t == nullptr || t->sizes() != sizes || t->scalar_type() != dt || t->device() != dev) return ok = false, nullptr;
        int64_t width = 1;
        for (size_t i = sizes.size(); i-- > 2;) {
            if (sizes[i] != 1 && t->stride(i) != width) return ok = false, nullptr;
            width *= sizes[i];
        }
        const int64_t d = sizes[1] > 1 ? t->stride(1) : sizes[0] > 1 ? t->stride(0) : width;
        if (d < width || d > 0x7fffffff || (sizes[0] > 1 && t->stride(0) != sizes[1] * d)) return ok = false, nullptr;
        ld = (int)d;
        return t->data_ptr();
    }
    int flag(PyObject *o) { return o == Py_True ? 1 : o == Py_False ? 0 : (ok = false, 0); }
    // a workspace of `need` bytes: the caller's, whose size the entry point checks, or a new one
    void *workspace(PyObject *o, size_t need, at::Tensor &ws, size_t &bytes) {
        if (!ok) return nullptr;
        if (o == Py_None) {
            ws = at::empty({(int64_t)(need > 16 ? need : 16)}, at::TensorOptions().dtype(at::kByte).device(dev));
        } else {
            const at::Tensor *t = plain(o);
            if (t == nullptr || t->device() != dev) return ok = false, nullptr;
            ws = *t;
        }
        bytes = ws.nbytes();
        return ws.data_ptr();
    }
};
// The call f, and what it wrote (None: not asked for) marked as changed in place: autograd then refuses a backward that has
// saved one of these tensors, a state that has been stepped on meanwhile, as after torch's own operations.
template <typename F> int unlocked(std::initializer_list<PyObject *> written, F f) {
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    if (st != 0) return st;
    for (PyObject *o : written) {
        if (o == Py_None) continue;
        c10::TensorImpl *t = THPVariable_Unpack(o).unsafeGetTensorImpl();
        if (!t->is_inference()) t->bump_version();
    }
    return st;
}

PyObject *py_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9 || g_layer.norm_fwd == nullptr) return not_taken();
    const double eps = PyFloat_AsDouble(a[8]);
    if (PyErr_Occurred()) return nullptr;
    try {
        const at::Tensor *x = Taker::tensor(a[0]);
        if (x == nullptr || x->dim() < 1) return not_taken();
        Taker k;
        k.lead(a[0], x->dim());
        const int64_t E = x->size(-1), rows = E > 0 ? x->numel() / E : 0;
        const at::IntArrayRef all = x->sizes(), lead = all.slice(0, all.size() - 1);
        if (!x->is_contiguous() || rows > 0x7fffffff) return not_taken();
        const float *gamma = k.f32(a[1], {E}, true), *beta = k.f32(a[2], {E}, true);
        void *y = k.mine(a[3], all), *s = k.mine(a[7], all, true);
        float *mean = k.f32(a[4], lead, true), *rstd = k.f32(a[5], lead, true);
        const void *r = k.mine(a[6], all, true), *px = x->data_ptr();
        if (!k.ok) return not_taken();
        void *q = stream();
        return PyLong_FromLong(unlocked({a[3], a[4], a[5], a[7]}, [&] { return g_layer.norm_fwd(px, r, gamma, beta, y, s, mean, rstd, (int)rows, (int)E, (float)eps, k.code, q); }));
    } catch (...) {
        return not_taken();
    }
}

PyObject *py_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 10 || g_layer.norm_bwd == nullptr) return not_taken();
    try {
        const at::Tensor *x = Taker::tensor(a[0]);
        if (x == nullptr || x->dim() < 1) return not_taken();
        Taker k;
        k.lead(a[0], x->dim());
        const int64_t E = x->size(-1), rows = E > 0 ? x->numel() / E : 0;
        const at::IntArrayRef all = x->sizes(), lead = all.slice(0, all.size() - 1);
        if (!x->is_contiguous() || rows > 0x7fffffff) return not_taken();
        const float *gamma = k.f32(a[1], {E}, true), *mean = k.f32(a[2], lead), *rstd = k.f32(a[3], lead);
        const void *dy = k.mine(a[4], all), *ds = k.mine(a[8], all, true), *px = x->data_ptr();
        void *dx = k.mine(a[5], all);
        float *dg = k.f32(a[6], {E}, true), *db = k.f32(a[7], {E}, true);
        if (!k.ok || (dg == nullptr && db == nullptr)) return not_taken();
        at::Tensor ws;
        size_t bytes = 0;
        void *w = k.workspace(a[9], g_layer.norm_bwd_ws((int)rows, (int)E, k.code), ws, bytes), *q = stream();
        if (!k.ok) return not_taken();
        return answer(unlocked({a[5], a[6], a[7]}, [&] { return g_layer.norm_bwd(px, gamma, mean, rstd, dy, ds, dx, dg, db, (int)rows, (int)E, k.code, w, bytes, q); }), a[9], ws);
    } catch (...) {
        return not_taken();
    }
}

// w [E, W]
bool taps(Taker &k, PyObject *o, int64_t E, int64_t &W, const float *&w) {
    const at::Tensor *t = Taker::tensor(o);
    if (t == nullptr || t->dim() != 2) return false;
    W = t->size(1);
    w = k.f32(o, {E, W});
    return k.ok && W >= 1 && W <= 0x7fffffff;
}

PyObject *py_conv_fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 8 || g_layer.conv_fwd == nullptr) return not_taken();
    try {
        Taker k;
        const at::Tensor *x = k.lead(a[0], 3);
        int64_t W;
        const float *w;
        if (x == nullptr || !taps(k, a[1], x->size(2), W, w)) return not_taken();
        const int64_t B = x->size(0), N = x->size(1), E = x->size(2);
        int ld;
        const void *px = k.rows(a[0], x->sizes(), ld), *x0 = k.mine(a[4], {B, W - 1, E}, true);
        const float *bias = k.f32(a[2], {E}, true);
        void *y = k.mine(a[3], {B, N, E}), *x1 = k.mine(a[5], {B, W - 1, E}, true);
        const int *len = static_cast<const int *>(k.dense(a[6], {B}, at::kInt, true));
        const int silu = k.flag(a[7]);
        if (!k.ok) return not_taken();
        void *q = stream();
        return PyLong_FromLong(unlocked({a[3], a[5]}, [&] { return g_layer.conv_fwd(px, ld, w, bias, x0, len, y, x1, (int)B, (int)N, (int)E, (int)W, silu, k.code, q); }));
    } catch (...) {
        return not_taken();
    }
}

PyObject *py_conv_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 13 || g_layer.conv_bwd == nullptr) return not_taken();
    try {
        Taker k;
        const at::Tensor *x = k.lead(a[0], 3);
        int64_t W;
        const float *w;
        if (x == nullptr || !taps(k, a[1], x->size(2), W, w)) return not_taken();
        const int64_t B = x->size(0), N = x->size(1), E = x->size(2);
        int ld;
        const void *px = k.rows(a[0], x->sizes(), ld), *dy = k.mine(a[3], {B, N, E});
        const float *bias = k.f32(a[2], {E}, true);
        void *dx = k.mine(a[4], {B, N, E});
        float *dw = k.f32(a[5], {E, W}, true), *db = k.f32(a[6], {E}, true);
        const void *x0 = k.mine(a[7], {B, W - 1, E}, true), *dx1 = k.mine(a[8], {B, W - 1, E}, true);
        void *dx0 = k.mine(a[9], {B, W - 1, E}, true);
        const int *len = static_cast<const int *>(k.dense(a[10], {B}, at::kInt, true));
        const int silu = k.flag(a[11]);
        if (!k.ok || (dw == nullptr && db == nullptr)) return not_taken();
        at::Tensor ws;
        size_t bytes = 0;
        void *s = k.workspace(a[12], g_layer.conv_bwd_ws((int)B, (int)N, (int)E, (int)W, k.code), ws, bytes), *q = stream();
        if (!k.ok) return not_taken();
        return answer(unlocked({a[4], a[5], a[6], a[9]}, [&] { return g_layer.conv_bwd(px, ld, w, bias, x0, len, dy, dx1, dx, dw, db, dx0, (int)B, (int)N, (int)E, (int)W, silu,
                                                             k.code, s, bytes, q); }), a[12], ws);
    } catch (...) {
        return not_taken();
    }
}

PyObject *py_conv_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 6 || g_layer.conv_step == nullptr) return not_taken();
    try {
        Taker k;
        const at::Tensor *x = k.lead(a[0], 2);
        int64_t W;
        const float *w;
        if (x == nullptr || !taps(k, a[1], x->size(1), W, w)) return not_taken();
        const int64_t B = x->size(0), E = x->size(1);
        const void *px = k.mine(a[0], {B, E});
        const float *bias = k.f32(a[2], {E}, true);
        void *state = k.mine(a[3], {B, W - 1, E}), *y = k.mine(a[4], {B, E});
        const int silu = k.flag(a[5]);
        if (!k.ok) return not_taken();
        void *q = stream();
        return PyLong_FromLong(unlocked({a[3], a[4]}, [&] { return g_layer.conv_step(px, w, bias, state, y, (int)B, (int)E, (int)W, silu, k.code, q); }));
    } catch (...) {
        return not_taken();
    }
}

// the inputs that a scan's forward and backward share
struct ScanIn {
    int64_t B, N, E, G, S;
    int ld[5];
    const void *x, *dt, *z, *Bt, *Ct;
    const float *A, *D, *bias, *h0;
    const int *len;
    bool take(Taker &k, PyObject *px, PyObject *pdt, PyObject *pA, PyObject *pB, PyObject *pC, PyObject *pD, PyObject *pz, PyObject *pbias,
              PyObject *ph0, PyObject *plen) {
        const at::Tensor *t = k.lead(px, 3), *bt = Taker::tensor(pB);
        if (t == nullptr || bt == nullptr || bt->dim() != 4 || !fits(*bt)) return false;
        B = t->size(0), N = t->size(1), E = t->size(2), G = bt->size(2), S = bt->size(3);
        if (G < 1 || S < 1 || E % G != 0) return false;
        x = k.rows(px, {B, N, E}, ld[0]), dt = k.rows(pdt, {B, N, E}, ld[1]), z = k.rows(pz, {B, N, E}, ld[2], true);
        Bt = k.rows(pB, {B, N, G, S}, ld[3]), Ct = k.rows(pC, {B, N, G, S}, ld[4]);
        A = k.f32(pA, {E, S}), D = k.f32(pD, {E}, true), bias = k.f32(pbias, {E}, true), h0 = k.f32(ph0, {B, E, S}, true);
        len = static_cast<const int *>(k.dense(plen, {B}, at::kInt, true));
        return k.ok;
    }
};

PyObject *py_scan_fwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 15 || g_layer.scan_fwd == nullptr) return not_taken();
    try {
        Taker k;
        ScanIn i;
        if (!i.take(k, a[0], a[1], a[2], a[3], a[4], a[6], a[7], a[8], a[9], a[11])) return not_taken();
        void *y = k.mine(a[5], {i.B, i.N, i.E});
        float *h1 = k.f32(a[10], {i.B, i.E, i.S}, true);
        const int flags = k.flag(a[12]) | 2 * k.flag(a[13]);
        at::Tensor ws;
        size_t bytes = 0;
        void *w = k.workspace(a[14], k.ok ? g_layer.scan_fwd_ws((int)i.B, (int)i.N, (int)i.E, (int)i.G, (int)i.S, k.code, flags) : 0, ws, bytes);
        if (!k.ok) return not_taken();
        void *q = stream();
        return answer(unlocked({a[5], a[10]}, [&] { return g_layer.scan_fwd(i.x, i.ld[0], i.dt, i.ld[1], i.z, i.ld[2], i.Bt, i.ld[3], i.Ct, i.ld[4], i.A, i.D, i.bias,
                                                             i.h0, i.len, y, h1, (int)i.B, (int)i.N, (int)i.E, (int)i.G, (int)i.S, flags, k.code, w,
                                                             bytes, q); }), a[14], ws);
    } catch (...) {
        return not_taken();
    }
}

PyObject *py_scan_bwd(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 24 || g_layer.scan_bwd == nullptr || a[22] == Py_None) return not_taken();
    try {
        Taker k;
        ScanIn i;
        if (!i.take(k, a[0], a[1], a[2], a[3], a[4], a[11], a[12], a[13], a[17], a[20])) return not_taken();
        const void *dy = k.mine(a[5], {i.B, i.N, i.E});
        void *dx = k.mine(a[6], {i.B, i.N, i.E}), *ddt = k.mine(a[7], {i.B, i.N, i.E}), *dz = k.mine(a[15], {i.B, i.N, i.E}, true);
        float *dA = k.f32(a[8], {i.E, i.S}), *dD = k.f32(a[14], {i.E}, true), *dbias = k.f32(a[16], {i.E}, true);
        void *dB = k.mine(a[9], {i.B, i.N, i.G, i.S}), *dC = k.mine(a[10], {i.B, i.N, i.G, i.S});
        const float *dh1 = k.f32(a[18], {i.B, i.E, i.S}, true);
        float *dh0 = k.f32(a[19], {i.B, i.E, i.S}, true);
        const int flags = k.flag(a[21]);
        const at::Tensor *fws = plain(a[22]);
        if (!k.ok || (i.z == nullptr) != (dz == nullptr) || fws == nullptr || fws->device() != k.dev ||
            fws->nbytes() < g_layer.scan_fwd_ws((int)i.B, (int)i.N, (int)i.E, (int)i.G, (int)i.S, k.code, flags | 2))
            return not_taken();
        at::Tensor ws;
        size_t bytes = 0;
        void *w = k.workspace(a[23], g_layer.scan_bwd_ws((int)i.B, (int)i.N, (int)i.E, (int)i.G, (int)i.S, k.code, flags | 2), ws, bytes);
        if (!k.ok) return not_taken();
        const void *fp = fws->data_ptr();
        void *q = stream();
        return answer(unlocked({a[6], a[7], a[8], a[9], a[10], a[14], a[15], a[16], a[19]}, [&] { return g_layer.scan_bwd(i.x, i.ld[0], i.dt, i.ld[1], i.z, i.ld[2], i.Bt, i.ld[3], i.Ct, i.ld[4], i.A, i.D, i.bias,
                                                             i.h0, i.len, fp, dy, dh1, dx, ddt, dz, dB, dC, dA, dD, dbias, dh0, (int)i.B, (int)i.N,
                                                             (int)i.E, (int)i.G, (int)i.S, flags, k.code, w, bytes, q); }), a[23], ws);
    } catch (...) {
        return not_taken();
    }
}

PyObject *py_scan_step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 11 || g_layer.scan_step == nullptr) return not_taken();
    try {
        Taker k;
        const at::Tensor *x = k.lead(a[0], 2), *bt = Taker::tensor(a[3]);
        if (x == nullptr || bt == nullptr || bt->dim() != 3 || !fits(*bt)) return not_taken();
        const int64_t B = x->size(0), E = x->size(1), G = bt->size(1), S = bt->size(2);
        if (G < 1 || S < 1 || E % G != 0) return not_taken();
        const void *px = k.mine(a[0], {B, E}), *dt = k.mine(a[1], {B, E}), *z = k.mine(a[8], {B, E}, true);
        const void *Bt = k.mine(a[3], {B, G, S}), *Ct = k.mine(a[4], {B, G, S});
        const float *A = k.f32(a[2], {E, S}), *D = k.f32(a[7], {E}, true), *bias = k.f32(a[9], {E}, true);
        float *h = k.f32(a[5], {B, E, S});
        void *y = k.mine(a[6], {B, E});
        const int flags = k.flag(a[10]);
        if (!k.ok) return not_taken();
        void *q = stream();
        return PyLong_FromLong(unlocked({a[5], a[6]}, [&] { return g_layer.scan_step(px, dt, z, Bt, Ct, A, D, bias, h, y, (int)B, (int)E, (int)G, (int)S, flags, k.code, q); }));
    } catch (...) {
        return not_taken();
    }
}

// bind_layer([12 addresses]): in the order of Layer
PyObject *py_bind_layer(PyObject *, PyObject *list) {
    static_assert(sizeof(Layer) == 12 * sizeof(void *), "one address each");
    if (!PyList_Check(list) || PyList_GET_SIZE(list) != 12) {
        PyErr_SetString(PyExc_ValueError, "12 addresses expected");
        return nullptr;
    }
    void *p[12];
    for (int i = 0; i < 12; ++i) {
        p[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&g_layer, p, sizeof(g_layer));
    Py_RETURN_NONE;
}

// bind([13 addresses]): step, fwd x 4, bwd x 4, fwd_ws x 2, bwd_ws x 2
PyObject *py_bind(PyObject *, PyObject *list) {
    if (!PyList_Check(list) || PyList_GET_SIZE(list) != 13) {
        PyErr_SetString(PyExc_ValueError, "13 addresses expected");
        return nullptr;
    }
    void *p[13];
    for (int i = 0; i < 13; ++i) {
        p[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
        if (PyErr_Occurred()) return nullptr;
    }
    g_step = reinterpret_cast<step_fn>(p[0]);
    for (int i = 0; i < 4; ++i) g_fwd[i] = reinterpret_cast<fwd_fn>(p[1 + i]), g_bwd[i] = reinterpret_cast<bwd_fn>(p[5 + i]);
    for (int i = 0; i < 2; ++i) g_fwd_ws[i] = reinterpret_cast<ws_fn>(p[9 + i]), g_bwd_ws[i] = reinterpret_cast<ws_fn>(p[11 + i]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_step)), METH_FASTCALL, nullptr},
    {"fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_fwd)), METH_FASTCALL, nullptr},
    {"bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_bwd)), METH_FASTCALL, nullptr},
    {"bind", py_bind, METH_O, nullptr},
#define LA_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
    LA_METHOD(norm_fwd), LA_METHOD(norm_bwd), LA_METHOD(conv_fwd), LA_METHOD(conv_bwd), LA_METHOD(conv_step),
    LA_METHOD(scan_fwd), LA_METHOD(scan_bwd), LA_METHOD(scan_step),
#undef LA_METHOD
    {"bind_layer", py_bind_layer, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
