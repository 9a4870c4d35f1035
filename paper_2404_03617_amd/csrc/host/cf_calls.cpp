// cf_calls.cpp -- calls of the training and scoring operators and of those for heads in native code
// (part of the module _cf_args): one function checks a call's arguments, makes
// its outputs with torch's allocator and calls the library on the current
// stream.  As with the checks of cf_args.cpp, these functions only say yes:
// with anything other than what a call wants they return None, and the
// binding's own path, which names what is wrong, takes over.  Where the
// library refuses they return its status.  Host time a call, through Python's
// checks and ctypes and through here, and what a call on little data takes:
// see the figures in training.py.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include "cf_native.h"
#include "convfirst.h"

namespace cfa {

namespace {

// The library's functions, given once it is loaded.
struct Library {
    decltype(&cf_layer_norm_forward) norm_forward;
    decltype(&cf_layer_norm_backward) norm_backward;
    decltype(&cf_layer_norm_backward_workspace_bytes) norm_ws;
    decltype(&cf_act_forward) act_forward;
    decltype(&cf_act_backward) act_backward;
    decltype(&cf_checkpoint_unpack) unpack;
    decltype(&cf_linear_weight_grad) wgrad;
    decltype(&cf_linear_weight_grad_workspace_bytes) wgrad_ws;
    decltype(&cf_log_probs_forward) log_probs;
    decltype(&cf_log_probs_workspace_bytes) log_probs_ws;
    decltype(&cf_log_probs_backward) log_probs_backward;
    decltype(&cf_group_norm_forward) group_norm;
    decltype(&cf_group_norm_workspace_bytes) group_norm_ws;
    decltype(&cf_group_norm_backward) group_norm_backward;
    decltype(&cf_group_norm_backward_workspace_bytes) group_norm_backward_ws;
    decltype(&cf_gated_ffn_forward) gated;
    decltype(&cf_gated_ffn_workspace_bytes) gated_ws;
    decltype(&cf_gated_ffn_backward) gated_backward;
    decltype(&cf_gated_ffn_backward_workspace_bytes) gated_backward_ws;
    decltype(&cf_linear_log_probs_forward) linear;
    decltype(&cf_linear_log_probs_workspace_bytes) linear_ws;
    decltype(&cf_linear_log_probs_backward) linear_backward;
    decltype(&cf_linear_log_probs_backward_workspace_bytes) linear_backward_ws;
};
Library lib;
bool bound = false;

// thrown where a call is not for this path
struct No {};

void must(bool ok) {
    if (!ok)
        throw No();
}

const at::Tensor &tensor(PyObject *o) {
    must(THPVariable_CheckExact(o));
    const at::Tensor &t = THPVariable_Unpack(o);
    must(t.defined());
    return t;
}

struct RowsOf {
    const at::Tensor *t;
    void *p;
    int64_t n, ld;
    int C, code;
};

// a tensor of rows whose dtype is one of the first `kinds` codes
RowsOf rows_of(PyObject *o, int kinds) {
    RowsOf r;
    r.t = &tensor(o);
    int64_t C;
    must(rows_view(*r.t, &r.n, &C, &r.ld, &r.code) && r.code < kinds && C >= 1 && C < ((int64_t)1 << 31));
    r.C = (int)C;
    r.p = r.t->data_ptr();
    return r;
}

// Address of a contiguous tensor of n * last elements on x's device, its last
// dimension of `last` (0: n elements in any shape); null for None.
template <typename P = void>
P *flat_of(PyObject *o, const at::Tensor &x, at::ScalarType type, int64_t n, int64_t last) {
    if (o == Py_None)
        return nullptr;
    const at::Tensor &t = tensor(o);
    must(plain(t) && t.scalar_type() == type && t.device() == x.device());
    must(last ? t.numel() == n * last && t.dim() >= 1 && t.size(t.dim() - 1) == last : t.numel() == n);
    return static_cast<P *>(t.data_ptr());
}
const float *floats(PyObject *o, const at::Tensor &x, int64_t n, int64_t last = 0) {
    return flat_of<const float>(o, x, at::kFloat, n, last);
}

at::Tensor fresh(const at::Tensor &x, at::IntArrayRef shape, at::ScalarType type) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(x.device()));
}

// x's leading dimensions and `last`
std::vector<int64_t> lead(const at::Tensor &x, int64_t last = -1) {
    std::vector<int64_t> s(x.sizes().begin(), x.sizes().end() - 1);
    if (last >= 0)
        s.push_back(last);
    return s;
}

at::ScalarType type_of(int code) { return code == 0 ? at::kHalf : code == 1 ? at::kBFloat16 : at::kFloat; }

// the caller's output, or a new one; its address and row stride
struct Out {
    at::Tensor t;
    void *p;
    int64_t ld;
};
Out out_of(PyObject *o, const at::Tensor &x, int code) {
    Out r;
    if (o == Py_None) {
        r.t = fresh(x, x.sizes(), type_of(code));
        r.ld = x.size(x.dim() - 1);
    } else {
        const RowsOf v = rows_of(o, 3);
        must(v.code == code && v.t->sizes() == x.sizes() && v.t->device() == x.device());
        r.t = *v.t;
        r.ld = v.ld;
    }
    r.p = r.t.data_ptr();
    return r;
}

int64_t blocks_of(int64_t C) { return (C + CF_CKPT_BLOCK - 1) / CF_CKPT_BLOCK; }

struct NewCheckpoint {
    at::Tensor q, scale;
    int8_t *qp = nullptr;
    float *sp = nullptr;
    void make(const at::Tensor &x, int64_t C) {
        q = fresh(x, x.sizes(), at::kChar);
        scale = fresh(x, lead(x, blocks_of(C)), at::kFloat);
        qp = static_cast<int8_t *>(q.data_ptr());
        sp = static_cast<float *>(scale.data_ptr());
    }
};

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

// a tensor to Python; None where there is none
PyObject *give(const at::Tensor &t) {
    if (!t.defined())
        Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
template <typename... Ts>
PyObject *give_all(const Ts &...ts) {
    constexpr int n = sizeof...(Ts);
    PyObject *items[n] = {give(ts)...}, *r = PyTuple_New(n);
    for (int i = 0; i < n; i++)
        PyTuple_SET_ITEM(r, i, items[i]);
    return r;
}

// Calls F on the argument tuple: None for what is not for this path, the
// status where the library refused.  No C++ exception leaves.
struct Refused {
    cf_status status;
};
void check(cf_status s) {
    if (s != CF_OK)
        throw Refused{s};
}
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (!bound)
        Py_RETURN_NONE;
    try {
        return F(args, n);
    } catch (const Refused &r) {
        return PyLong_FromLong(r.status);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    must(v >= 0);
    return v != 0;
}
float real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    must(!(v == -1.0 && PyErr_Occurred()));
    return (float)v;
}
long whole(PyObject *o) {
    const long v = PyLong_AsLong(o);
    must(!(v == -1 && PyErr_Occurred()));
    return v;
}

// (x, weight, bias, eps, out) -> y
PyObject *norm_forward(PyObject *const *a, Py_ssize_t n) {
    must(n == 5);
    const RowsOf x = rows_of(a[0], 2);
    const float *w = floats(a[1], *x.t, x.C), *b = floats(a[2], *x.t, x.C), eps = real(a[3]);
    const Out y = out_of(a[4], *x.t, x.code);
    check(lib.norm_forward(x.p, y.p, w, b, nullptr, nullptr, nullptr, x.n, x.C, x.ld, y.ld, eps, (cf_dtype)x.code,
                           stream()));
    return give(y.t);
}

// (x, weight, bias, eps, checkpoint, out) -> (y, stats, q, scale)
PyObject *norm_forward_save(PyObject *const *a, Py_ssize_t n) {
    must(n == 6);
    const RowsOf x = rows_of(a[0], 2);
    const float *w = floats(a[1], *x.t, x.C), *b = floats(a[2], *x.t, x.C), eps = real(a[3]);
    const Out y = out_of(a[5], *x.t, x.code);
    const at::Tensor stats = fresh(*x.t, lead(*x.t, 2), at::kFloat);
    NewCheckpoint ck;
    if (truth(a[4]))
        ck.make(*x.t, x.C);
    check(lib.norm_forward(x.p, y.p, w, b, static_cast<float *>(stats.data_ptr()), ck.qp, ck.sp, x.n, x.C, x.ld, y.ld,
                           eps, (cf_dtype)x.code, stream()));
    return give_all(y.t, stats, ck.q, ck.scale);
}

// (dy, x or None, q, scale, stats, weight, param_grads, out) -> (dx, dweight, dbias)
PyObject *norm_backward(PyObject *const *a, Py_ssize_t n) {
    must(n == 8);
    const RowsOf dy = rows_of(a[0], 2);
    RowsOf x = dy;
    x.p = nullptr;
    const int8_t *q = nullptr;
    const float *scale = nullptr;
    if (a[1] == Py_None) {
        must(a[2] != Py_None && a[3] != Py_None);
        q = flat_of<const int8_t>(a[2], *dy.t, at::kChar, dy.n, dy.C);
        scale = floats(a[3], *dy.t, dy.n, blocks_of(dy.C));
    } else {
        x = rows_of(a[1], 2);
        must(x.code == dy.code && x.t->sizes() == dy.t->sizes() && x.t->device() == dy.t->device());
    }
    must(a[4] != Py_None);
    const float *stats = floats(a[4], *dy.t, dy.n, 2), *w = floats(a[5], *dy.t, dy.C);
    const Out dx = out_of(a[7], *dy.t, dy.code);
    at::Tensor dw, db, ws;
    size_t bytes = 0;
    if (truth(a[6])) {
        dw = fresh(*dy.t, {dy.C}, at::kFloat);
        db = fresh(*dy.t, {dy.C}, at::kFloat);
        bytes = lib.norm_ws(dy.n, dy.C);
        if (bytes)
            ws = fresh(*dy.t, {(int64_t)bytes}, at::kByte);
    }
    check(lib.norm_backward(dy.p, x.p, q, scale, stats, w, dx.p, dw.defined() ? static_cast<float *>(dw.data_ptr()) : nullptr,
                            db.defined() ? static_cast<float *>(db.data_ptr()) : nullptr,
                            ws.defined() ? ws.data_ptr() : nullptr, bytes, dy.n, dy.C, dy.ld, x.ld, dx.ld,
                            (cf_dtype)dy.code, stream()));
    return give_all(dx.t, dw, db);
}

// (u, act, with h, checkpoint of u, checkpoint of h, out) -> (h, qu, scale_u, qh, scale_h)
PyObject *act_forward(PyObject *const *a, Py_ssize_t n) {
    must(n == 6);
    const RowsOf u = rows_of(a[0], 2);
    const long act = whole(a[1]);
    Out h{at::Tensor(), nullptr, u.C};
    if (truth(a[2]))
        h = out_of(a[5], *u.t, u.code);
    NewCheckpoint cu, ch;
    if (truth(a[3]))
        cu.make(*u.t, u.C);
    if (truth(a[4]))
        ch.make(*u.t, u.C);
    check(lib.act_forward(u.p, h.p, cu.qp, cu.sp, ch.qp, ch.sp, u.n, u.C, u.ld, h.ld, (cf_dtype)u.code, (cf_act)act,
                          stream()));
    return give_all(h.t, cu.q, cu.scale, ch.q, ch.scale);
}

// (dh, q, scale, act, out) -> du
PyObject *act_backward(PyObject *const *a, Py_ssize_t n) {
    must(n == 5 && a[1] != Py_None && a[2] != Py_None);
    const RowsOf dh = rows_of(a[0], 2);
    const int8_t *q = flat_of<const int8_t>(a[1], *dh.t, at::kChar, dh.n, dh.C);
    const float *scale = floats(a[2], *dh.t, dh.n, blocks_of(dh.C));
    const long act = whole(a[3]);
    const Out du = out_of(a[4], *dh.t, dh.code);
    check(lib.act_backward(dh.p, q, scale, du.p, dh.n, dh.C, dh.ld, du.ld, (cf_dtype)dh.code, (cf_act)act, stream()));
    return give(du.t);
}

// a checkpoint's q: rows and channels
RowsOf checkpoint_rows(PyObject *o) {
    RowsOf q;
    q.t = &tensor(o);
    must(plain(*q.t) && q.t->scalar_type() == at::kChar && q.t->dim() >= 1);
    const int64_t C = q.t->size(q.t->dim() - 1);
    must(C >= 1 && C < ((int64_t)1 << 31));
    q.C = (int)C;
    q.n = q.t->numel() / C;
    q.ld = C;
    q.code = 3;
    q.p = q.t->data_ptr();
    return q;
}

// (q, scale, dtype code, out) -> x
PyObject *unpack(PyObject *const *a, Py_ssize_t n) {
    must(n == 4 && a[1] != Py_None);
    const RowsOf q = checkpoint_rows(a[0]);
    const float *scale = floats(a[1], *q.t, q.n, blocks_of(q.C));
    const long code = whole(a[2]);
    const Out x = out_of(a[3], *q.t, (int)code);
    check(lib.unpack(static_cast<const int8_t *>(q.p), scale, x.p, q.n, q.C, x.ld, (cf_dtype)code, stream()));
    return give(x.t);
}

// (dy, q, scale, stats, weight, bias) -> (dw, db)
PyObject *wgrad(PyObject *const *a, Py_ssize_t n) {
    must(n == 6 && a[2] != Py_None);
    const RowsOf dy = rows_of(a[0], 2), q = checkpoint_rows(a[1]);
    must(q.n == dy.n && q.t->device() == dy.t->device());
    const float *scale = floats(a[2], *dy.t, dy.n, blocks_of(q.C)), *stats = floats(a[3], *dy.t, dy.n, 2);
    const float *w = floats(a[4], *dy.t, q.C), *b = floats(a[5], *dy.t, q.C);
    const at::Tensor dw = fresh(*dy.t, {dy.C, q.C}, type_of(dy.code)), db = fresh(*dy.t, {dy.C}, at::kFloat);
    const size_t bytes = lib.wgrad_ws(dy.n, dy.C, q.C);
    at::Tensor ws;
    if (bytes)
        ws = fresh(*dy.t, {(int64_t)bytes}, at::kByte);
    check(lib.wgrad(dy.p, static_cast<const int8_t *>(q.p), scale, stats, w, b, dw.data_ptr(),
                    static_cast<float *>(db.data_ptr()), bytes ? ws.data_ptr() : nullptr, bytes, dy.n, dy.C, q.C,
                    dy.ld, (cf_dtype)dy.code, stream()));
    return give_all(dw, db);
}

// (logits, tokens or None, top) -> (logp, entropy, stats, top_logp, top_ids)
PyObject *log_probs(PyObject *const *a, Py_ssize_t n) {
    must(n == 3);
    const RowsOf z = rows_of(a[0], 3);
    const int64_t *tokens = flat_of<const int64_t>(a[1], *z.t, at::kLong, z.n, 0);
    const long top = whole(a[2]);
    must(top >= 0 && top <= CF_TOP_MAX && top <= z.C);
    const std::vector<int64_t> shape = lead(*z.t);
    at::Tensor logp, top_logp, top_ids, ws;
    if (tokens || a[1] != Py_None)
        logp = fresh(*z.t, shape, at::kFloat);
    const at::Tensor entropy = fresh(*z.t, shape, at::kFloat), stats = fresh(*z.t, lead(*z.t, 2), at::kFloat);
    if (top) {
        top_logp = fresh(*z.t, lead(*z.t, top), at::kFloat);
        top_ids = fresh(*z.t, lead(*z.t, top), at::kLong);
    }
    const size_t bytes = lib.log_probs_ws(z.n, z.C, (int)top);
    if (bytes)
        ws = fresh(*z.t, {(int64_t)bytes}, at::kByte);
    check(lib.log_probs(z.p, tokens, logp.defined() ? static_cast<float *>(logp.data_ptr()) : nullptr,
                        static_cast<float *>(entropy.data_ptr()), static_cast<float *>(stats.data_ptr()),
                        top ? static_cast<float *>(top_logp.data_ptr()) : nullptr,
                        top ? static_cast<int64_t *>(top_ids.data_ptr()) : nullptr, (int)top,
                        bytes ? ws.data_ptr() : nullptr, bytes, z.n, z.C, z.ld, (cf_logits_dtype)z.code, stream()));
    return give_all(logp, entropy, stats, top_logp, top_ids);
}

// (logits, tokens, stats, entropy, d_logp, d_entropy, out) -> dlogits
PyObject *log_probs_backward(PyObject *const *a, Py_ssize_t n) {
    must(n == 7 && a[2] != Py_None && a[3] != Py_None);
    const RowsOf z = rows_of(a[0], 3);
    const int64_t *tokens = flat_of<const int64_t>(a[1], *z.t, at::kLong, z.n, 0);
    const float *stats = floats(a[2], *z.t, z.n, 2), *entropy = floats(a[3], *z.t, z.n);
    const float *gl = floats(a[4], *z.t, z.n), *gh = floats(a[5], *z.t, z.n);
    const Out dz = out_of(a[6], *z.t, z.code);
    check(lib.log_probs_backward(z.p, tokens, stats, entropy, gl, gh, dz.p, z.n, z.C, z.ld, dz.ld,
                                 (cf_logits_dtype)z.code, stream()));
    return give(dz.t);
}

// --- operators for heads ----------------------------------------------------

// These run on their tensors' device: this path is for the current one.
void on_current(const at::Tensor &x) { must(x.device().index() == c10::hip::current_device()); }

float *data(const at::Tensor &t) { return t.defined() ? static_cast<float *>(t.data_ptr()) : nullptr; }

struct Workspace {
    at::Tensor t;
    void *p = nullptr;
    size_t bytes = 0;
    Workspace(const at::Tensor &x, size_t n) : bytes(n) {
        if (n) {
            t = fresh(x, {(int64_t)n}, at::kByte);
            p = t.data_ptr();
        }
    }
};

// feature maps [N, .., C]: images and their pixels
RowsOf images_of(PyObject *o, int64_t *N, int64_t *P) {
    const RowsOf x = rows_of(o, 2);
    must(x.t->dim() >= 2);
    *N = x.t->size(0);
    *P = *N ? x.n / *N : 0;
    return x;
}

// (x, groups, weight, bias, eps, act, save, out) -> (y, stats or None)
PyObject *group_norm(PyObject *const *a, Py_ssize_t n) {
    must(n == 8 && PyLong_CheckExact(a[1]));
    int64_t N, P;
    const RowsOf x = images_of(a[0], &N, &P);
    on_current(*x.t);
    const long G = whole(a[1]), act = whole(a[5]);
    must(G >= 1 && G <= x.C && x.C % G == 0);
    const float *w = floats(a[2], *x.t, x.C), *b = floats(a[3], *x.t, x.C), eps = real(a[4]);
    const Out y = out_of(a[7], *x.t, x.code);
    at::Tensor stats;
    if (truth(a[6]))
        stats = fresh(*x.t, {N, G, 2}, at::kFloat);
    const Workspace ws(*x.t, lib.group_norm_ws(N, P, x.C, (int)G));
    check(lib.group_norm(x.p, y.p, w, b, data(stats), ws.p, ws.bytes, N, P, x.C, (int)G, x.ld, y.ld, eps,
                         (cf_dtype)x.code, (cf_act)act, stream()));
    return give_all(y.t, stats);
}

// (dy, x, stats, weight, bias, act, param_grads, out) -> (dx, dweight, dbias)
PyObject *group_norm_backward(PyObject *const *a, Py_ssize_t n) {
    must(n == 8);
    int64_t N, P;
    const RowsOf dy = images_of(a[0], &N, &P), x = rows_of(a[1], 2);
    on_current(*dy.t);
    must(x.code == dy.code && x.t->sizes() == dy.t->sizes() && x.t->device() == dy.t->device());
    const at::Tensor &st = tensor(a[2]);
    must(st.dim() == 3 && st.size(1) >= 1 && st.size(1) <= dy.C && dy.C % st.size(1) == 0);
    const int G = (int)st.size(1);
    const float *stats = floats(a[2], *dy.t, N * G, 2), *w = floats(a[3], *dy.t, dy.C), *b = floats(a[4], *dy.t, dy.C);
    const long act = whole(a[5]);
    const Out dx = out_of(a[7], *dy.t, dy.code);
    at::Tensor dw, db;
    if (truth(a[6])) {
        dw = fresh(*dy.t, {dy.C}, at::kFloat);
        db = fresh(*dy.t, {dy.C}, at::kFloat);
    }
    const Workspace ws(*dy.t, lib.group_norm_backward_ws(N, P, dy.C, G));
    check(lib.group_norm_backward(dy.p, x.p, stats, w, b, dx.p, data(dw), data(db), ws.p, ws.bytes, N, P, dy.C, G, dy.ld,
                                  x.ld, dx.ld, (cf_dtype)dy.code, (cf_act)act, stream()));
    return give_all(dx.t, dw, db);
}

// a weight matrix [rows (-1: any), cols] of x's type and device
RowsOf matrix_of(PyObject *o, const RowsOf &x, int64_t rows, int64_t cols) {
    const RowsOf w = rows_of(o, 2);
    must(w.t->dim() == 2 && w.code == x.code && w.C == cols && (rows < 0 ? w.n >= 1 : w.n == rows) &&
         w.n < ((int64_t)1 << 31) && w.t->device() == x.t->device());
    return w;
}

// whether the products read these rows in place
bool readable(const RowsOf &r) { return ((uintptr_t)r.p & 15) == 0 && r.ld % 8 == 0 && r.ld < ((int64_t)1 << 22); }

// (x, w_gate, w_up, w_down, act, save, out) -> (y, saved or None)
PyObject *gated(PyObject *const *a, Py_ssize_t n) {
    must(n == 7);
    const RowsOf x = rows_of(a[0], 2);
    on_current(*x.t);
    const RowsOf g = matrix_of(a[1], x, -1, x.C), u = matrix_of(a[2], x, g.n, x.C), d = matrix_of(a[3], x, x.C, g.n);
    const int H = (int)g.n;
    const long act = whole(a[4]);
    const Out y = out_of(a[6], *x.t, x.code);
    at::Tensor saved;
    if (truth(a[5]))
        saved = fresh(*x.t, lead(*x.t, 2 * (int64_t)H), at::kFloat);
    const bool plain = readable(x) && readable(g) && readable(u) && readable(d) && g.ld == u.ld;
    const Workspace ws(*x.t, lib.gated_ws(x.n, x.C, H, plain));
    check(lib.gated(x.p, g.p, u.p, d.p, y.p, data(saved), ws.p, ws.bytes, x.n, x.C, H, x.ld, g.ld, u.ld, d.ld, y.ld,
                    (cf_dtype)x.code, (cf_act)act, stream()));
    return give_all(y.t, saved);
}

// (dy, x, saved, w_gate, w_up, w_down, act, out) -> (dx, dw_gate, dw_up, dw_down)
PyObject *gated_backward(PyObject *const *a, Py_ssize_t n) {
    must(n == 8 && a[2] != Py_None);
    const RowsOf dy = rows_of(a[0], 2), x = rows_of(a[1], 2);
    on_current(*dy.t);
    must(x.code == dy.code && x.t->sizes() == dy.t->sizes() && x.t->device() == dy.t->device());
    const RowsOf g = matrix_of(a[3], dy, -1, dy.C), u = matrix_of(a[4], dy, g.n, dy.C), d = matrix_of(a[5], dy, dy.C, g.n);
    const int H = (int)g.n;
    const float *saved = floats(a[2], *dy.t, dy.n, 2 * (int64_t)H);
    const long act = whole(a[6]);
    const Out dx = out_of(a[7], *dy.t, dy.code);
    const at::ScalarType type = type_of(dy.code);
    const at::Tensor dg = fresh(*dy.t, {H, dy.C}, type), du = fresh(*dy.t, {H, dy.C}, type),
                     dd = fresh(*dy.t, {dy.C, H}, type);
    const bool plain = readable(dy) && readable(x) && readable(g) && readable(u) && readable(d) && g.ld == u.ld;
    const Workspace ws(*dy.t, lib.gated_backward_ws(dy.n, dy.C, H, plain));
    check(lib.gated_backward(dy.p, x.p, saved, g.p, u.p, d.p, dx.p, dg.data_ptr(), du.data_ptr(), dd.data_ptr(), ws.p,
                             ws.bytes, dy.n, dy.C, H, dy.ld, x.ld, g.ld, u.ld, d.ld, dx.ld, (cf_dtype)dy.code,
                             (cf_act)act, stream()));
    return give_all(dx.t, dg, du, dd);
}

// (x, weight, tokens or None) -> (logp or None, lse)
PyObject *linear(PyObject *const *a, Py_ssize_t n) {
    must(n == 3);
    const RowsOf x = rows_of(a[0], 2);
    on_current(*x.t);
    const RowsOf w = matrix_of(a[1], x, -1, x.C);
    const int64_t *tokens = flat_of<const int64_t>(a[2], *x.t, at::kLong, x.n, 0);
    const std::vector<int64_t> shape = lead(*x.t);
    at::Tensor logp;
    if (a[2] != Py_None)
        logp = fresh(*x.t, shape, at::kFloat);
    const at::Tensor lse = fresh(*x.t, shape, at::kFloat);
    const Workspace ws(*x.t, lib.linear_ws(x.n, x.C, (int)w.n, readable(x) && readable(w)));
    check(lib.linear(x.p, w.p, tokens, data(logp), data(lse), ws.p, ws.bytes, x.n, x.C, (int)w.n, x.ld, w.ld,
                     (cf_dtype)x.code, stream()));
    return give_all(logp, lse);
}

// (x, weight, tokens or None, logp or None, lse, d_logp, d_lse, out) -> (dx, dweight)
PyObject *linear_backward(PyObject *const *a, Py_ssize_t n) {
    must(n == 8 && a[4] != Py_None);
    const RowsOf x = rows_of(a[0], 2);
    on_current(*x.t);
    const RowsOf w = matrix_of(a[1], x, -1, x.C);
    const int64_t *tokens = flat_of<const int64_t>(a[2], *x.t, at::kLong, x.n, 0);
    const float *logp = floats(a[3], *x.t, x.n), *lse = floats(a[4], *x.t, x.n);
    const float *gl = floats(a[5], *x.t, x.n), *gs = floats(a[6], *x.t, x.n);
    const Out dx = out_of(a[7], *x.t, x.code);
    const at::Tensor dw = fresh(*x.t, {w.n, x.C}, type_of(x.code));
    const Workspace ws(*x.t, lib.linear_backward_ws(x.n, x.C, (int)w.n, readable(x) && readable(w)));
    check(lib.linear_backward(x.p, w.p, tokens, logp, lse, gl, gs, dx.p, dw.data_ptr(), ws.p, ws.bytes, x.n, x.C,
                              (int)w.n, x.ld, w.ld, dx.ld, (cf_dtype)x.code, stream()));
    return give_all(dx.t, dw);
}

// bind((address, ..)): the library's functions, in the order of Library
PyObject *bind(PyObject *, PyObject *arg) {
    constexpr Py_ssize_t n = sizeof(Library) / sizeof(void *);
    if (!PyTuple_CheckExact(arg) || PyTuple_GET_SIZE(arg) != n) {
        PyErr_SetString(PyExc_ValueError, "bind: a tuple of the library's functions");
        return nullptr;
    }
    void *p[n];
    for (Py_ssize_t i = 0; i < n; i++) {
        p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(arg, i));
        if (!p[i]) {
            if (!PyErr_Occurred())
                PyErr_SetString(PyExc_ValueError, "bind: a null function");
            return nullptr;
        }
    }
    memcpy(&lib, p, sizeof lib);
    bound = true;
    Py_RETURN_NONE;
}

#define CF_CALL(name, f) \
    { name, (PyCFunction)(void (*)(void))call<f>, METH_FASTCALL, nullptr }

}  // namespace

PyMethodDef calls[] = {CF_CALL("norm_forward", norm_forward),
                       CF_CALL("norm_forward_save", norm_forward_save),
                       CF_CALL("norm_backward", norm_backward),
                       CF_CALL("act_forward", act_forward),
                       CF_CALL("act_backward", act_backward),
                       CF_CALL("unpack", unpack),
                       CF_CALL("wgrad", wgrad),
                       CF_CALL("log_probs", log_probs),
                       CF_CALL("log_probs_backward", log_probs_backward),
                       CF_CALL("group_norm", group_norm),
                       CF_CALL("group_norm_backward", group_norm_backward),
                       CF_CALL("gated", gated),
                       CF_CALL("gated_backward", gated_backward),
                       CF_CALL("linear", linear),
                       CF_CALL("linear_backward", linear_backward),
                       {"bind", bind, METH_O, nullptr},
                       {nullptr, nullptr, 0, nullptr}};

}  // namespace cfa
