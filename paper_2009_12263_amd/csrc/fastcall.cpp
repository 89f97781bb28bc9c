// Native argument marshalling of the Python binding (binding.py): the calls that programs make in earnest, device tensors
// in plain descriptions, go from here straight to the C ABI.  Everything else (no tensor, other tensor classes,
// descriptions that do not fit their tensors, integers of other types) returns -1 before anything is launched, and the
// binding marshals it itself, with its own checks and messages.
//
// Why: a call of a small product is bound by the host.  With the descriptors built in Python and ctypes the
// marshalling took 4 to 5 us of the 7 to 9 of a call of fg_gemm and 8 of the 11 to 12 of fg_contract; the launch itself takes 3.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <pthread.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/flexgemm.h"

namespace {

typedef fg_status (*GemmFn)(int64_t, int64_t, int64_t, float, const fg_matrix *, const fg_matrix *, float, const fg_matrix *, const fg_matrix *,
                            const fg_epilogue *, void *);
typedef fg_status (*GemmExFn)(int64_t, int64_t, int64_t, float, const fg_matrix *, const fg_matrix *, float, const fg_matrix *, const fg_matrix *,
                              const fg_epilogue *, const fg_load_transforms *, void *);
typedef fg_status (*DualFn)(int64_t, int64_t, int64_t, float, const fg_matrix *, const fg_matrix *, float, const fg_matrix *, const fg_matrix *, void *);
typedef fg_status (*ContractFn)(int32_t, const int32_t *, const int64_t *, const void *, int32_t, const int32_t *, const int64_t *, const void *, int32_t,
                                const int32_t *, const int64_t *, const float *, float *, int32_t, const int32_t *, const int64_t *, float, float, void *);

struct Entry { GemmFn gemm; GemmExFn ex, noalloc; DualFn dual; ContractFn contract; } g_entry;
PyObject *g_matrix_type, *g_raw_stream, *g_device;                 // binding.Matrix and how the current stream is asked for
PyObject *s_re, *s_im, *s_layout, *s_ld, *s_dtype;
bool g_forked;                                                    // a child of fork() cannot use the GPU: torch says so

// An integer that fits; anything else is left to the binding.
bool as_int(PyObject *o, int64_t &v) {
    if (!o || !PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool as_float(PyObject *o, float &v) {
    if (PyFloat_CheckExact(o)) { v = (float)PyFloat_AS_DOUBLE(o); return true; }
    int64_t i;
    if (!as_int(o, i) || i > (1 << 24) || i < -(1 << 24)) return false;
    v = (float)i;
    return true;
}

// Address and element count of a plain device tensor; what its dtype is called in the C ABI.
struct Device { void *ptr; int64_t numel; int dtype; bool is_complex; };
bool device_tensor(PyObject *o, Device &d) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) return false;
    d.ptr = t.data_ptr();
    d.numel = t.numel();
    d.is_complex = t.is_complex();
    switch (t.scalar_type()) {
        case at::kHalf: d.dtype = FG_F16; break;
        case at::kBFloat16: d.dtype = FG_BF16; break;
        case at::kFloat: d.dtype = FG_F32; break;
        case at::kComplexHalf: d.dtype = FG_CF16; break;
        case at::kComplexFloat: d.dtype = FG_CF32; break;
        default: return false;
    }
    return true;
}

// binding.Matrix -> fg_matrix, with the binding's check that the tensors hold the matrix.  present: false for None.
bool matrix(PyObject *o, int64_t rows, int64_t cols, fg_matrix &x, bool &present) {
    present = o != Py_None;
    if (!present) return true;
    if ((PyObject *)Py_TYPE(o) != g_matrix_type) return false;
    PyObject **dict = _PyObject_GetDictPtr(o);
    if (!dict || !*dict) return false;
    PyObject *re = PyDict_GetItemWithError(*dict, s_re), *im = PyDict_GetItemWithError(*dict, s_im), *dt = PyDict_GetItemWithError(*dict, s_dtype);
    int64_t layout, ld, dtype;
    if (!re || !im || !dt || !as_int(PyDict_GetItemWithError(*dict, s_layout), layout) || !as_int(PyDict_GetItemWithError(*dict, s_ld), ld)) return false;
    Device t[2];
    if (!device_tensor(re, t[0])) return false;
    const bool two = im != Py_None;
    if (two && !device_tensor(im, t[1])) return false;
    if (dt == Py_None) dtype = t[0].dtype;
    else if (!as_int(dt, dtype)) return false;
    if (layout < 0 || layout > FG_ZERO || dtype < 0 || dtype > FG_CF32 || ld < 0 || ld > (1ll << 31) || rows > (1 << 30) || cols > (1 << 30)) return false;
    const int64_t need = layout == FG_COL ? (ld >= rows ? (cols - 1) * ld + rows : 0) : layout == FG_ROW ? (ld >= cols ? (rows - 1) * ld + cols : 0)
                       : layout == FG_DIAG ? (rows < cols ? rows : cols) : 0;
    for (int k = 0; k < (two ? 2 : 1); ++k) {
        const int64_t per_entry = (dt != Py_None && (dtype == FG_CF16 || dtype == FG_CF32) && !t[k].is_complex) ? 2 : 1;
        if (need > t[k].numel / per_entry) return false;              // the binding raises
    }
    x.re = t[0].ptr;
    x.im = two ? t[1].ptr : nullptr;
    x.dtype = (int32_t)dtype;
    x.layout = (int32_t)layout;
    x.ld = ld;
    return true;
}

bool current_stream(PyObject *stream, void *&handle) {
    if (stream != Py_None) return false;
    PyObject *dev = PyObject_CallNoArgs(g_device);
    PyObject *raw = dev ? PyObject_CallOneArg(g_raw_stream, dev) : nullptr;
    Py_XDECREF(dev);
    handle = raw ? PyLong_AsVoidPtr(raw) : nullptr;
    Py_XDECREF(raw);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

PyObject *not_here() {
    PyErr_Clear();
    return PyLong_FromLong(-1);
}

// gemm(M, N, K, alpha, A, B, beta, C, D, bias, bias_dim, act, stream, a_add, b_add, c_act, noalloc) -> status
// dual(M, N, K, alpha, A, B, beta, C, D, stream) -> status
PyObject *product(PyObject *const *a, Py_ssize_t n, bool dual) {
    if (g_forked || n != (dual ? 10 : 17)) return not_here();
    try {
        int64_t M, N, K, bias_dim = 0, act = 0, c_act = 0;
        float alpha, beta, a_add = 0.f, b_add = 0.f;
        if (!as_int(a[0], M) || !as_int(a[1], N) || !as_int(a[2], K) || !as_float(a[3], alpha) || !as_float(a[6], beta) || M <= 0 || N <= 0 || K <= 0) return not_here();
        fg_matrix A, B, C, D;
        bool has_a, has_b, has_c, has_d;
        if (!matrix(a[4], M, K, A, has_a) || !matrix(a[5], K, N, B, has_b) || !matrix(a[7], M, N, C, has_c) || !matrix(a[8], M, N, D, has_d)) return not_here();
        if (!has_a || !has_b || !has_d) return not_here();
        fg_epilogue ep = {};
        bool has_ep = false, noalloc = false;
        if (!dual) {
            if (!as_int(a[10], bias_dim) || !as_int(a[11], act) || !as_float(a[13], a_add) || !as_float(a[14], b_add) || !as_int(a[15], c_act) ||
                (a[16] != Py_False && a[16] != Py_True)) return not_here();
            if (bias_dim < 0 || bias_dim > 1 || act < 0 || act > 1 || c_act < 0 || c_act > 1) return not_here();
            noalloc = a[16] == Py_True;
            if (a[9] != Py_None) {
                Device bias;
                if (!device_tensor(a[9], bias)) return not_here();
                ep.bias = (const float *)bias.ptr;
            }
            ep.bias_dim = (int32_t)bias_dim;
            ep.act = (int32_t)act;
            has_ep = ep.bias || act != FG_ACT_NONE || a[9] != Py_None;
        }
        void *stream;
        if (!current_stream(a[dual ? 9 : 12], stream)) return not_here();
        const fg_matrix *c = has_c ? &C : nullptr;
        const fg_epilogue *e = has_ep ? &ep : nullptr;
        const fg_load_transforms lt = {a_add, b_add, (int32_t)c_act};
        auto call = [&]() noexcept {
            if (dual) return g_entry.dual(M, N, K, alpha, &A, &B, beta, c, &D, stream);
            if (noalloc) return g_entry.noalloc(M, N, K, alpha, &A, &B, beta, c, &D, e, &lt, stream);
            if (a_add != 0.f || b_add != 0.f || c_act != FG_ACT_NONE) return g_entry.ex(M, N, K, alpha, &A, &B, beta, c, &D, e, &lt, stream);
            return g_entry.gemm(M, N, K, alpha, &A, &B, beta, c, &D, e, stream);
        };
        fg_status st;
        Py_BEGIN_ALLOW_THREADS
        st = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(st);
    } catch (...) {                                                  // a tensor without storage: the binding's own call says what is wrong
        return not_here();
    }
}
PyObject *gemm(PyObject *, PyObject *const *args, Py_ssize_t n) { return product(args, n, false); }
PyObject *dual(PyObject *, PyObject *const *args, Py_ssize_t n) { return product(args, n, true); }

constexpr int kModes = 12, kLabels = 24;                              // what the library takes
struct Modes { int32_t n; int32_t label[kModes]; int64_t stride[kModes]; };
bool modes(PyObject *labels, PyObject *strides, Modes &m) {
    if (!(PyList_CheckExact(labels) || PyTuple_CheckExact(labels)) || !(PyList_CheckExact(strides) || PyTuple_CheckExact(strides))) return false;
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(labels);
    if (n > kModes || PySequence_Fast_GET_SIZE(strides) != n) return false;
    for (Py_ssize_t i = 0; i < n; ++i) {
        int64_t l, s;
        if (!as_int(PySequence_Fast_GET_ITEM(labels, i), l) || !as_int(PySequence_Fast_GET_ITEM(strides, i), s)) return false;
        if (l < INT32_MIN || l > INT32_MAX || s < 0 || s > (1ll << 40)) return false;
        m.label[i] = (int32_t)l;
        m.stride[i] = s;
    }
    m.n = (int32_t)n;
    return true;
}

// contract(modesA, stridesA, A, modesB, stridesB, B, modesC, stridesC, Cin, Cout, extents, alpha, beta, stream) -> status
PyObject *contract(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (g_forked || n != 14) return not_here();
    try {
        Modes mA, mB, mC;
        Device A, B, Cin = {}, Cout;
        float alpha, beta;
        if (!modes(a[0], a[1], mA) || !modes(a[3], a[4], mB) || !modes(a[6], a[7], mC) || !PyDict_CheckExact(a[10])) return not_here();
        if (!device_tensor(a[2], A) || !device_tensor(a[5], B) || !device_tensor(a[9], Cout)) return not_here();
        if (a[8] != Py_None && !device_tensor(a[8], Cin)) return not_here();
        if (!as_float(a[11], alpha) || !as_float(a[12], beta)) return not_here();
        int32_t labels[kLabels], count = 0;
        int64_t extents[kLabels];
        PyObject *key, *value;
        Py_ssize_t pos = 0;
        while (PyDict_Next(a[10], &pos, &key, &value)) {
            int64_t l, e;
            if (count == kLabels || !as_int(key, l) || !as_int(value, e) || l < INT32_MIN || l > INT32_MAX || e <= 0 || e > (1 << 30)) return not_here();
            labels[count] = (int32_t)l;
            extents[count++] = e;
        }
        // the last element that a description reaches must exist (a mode without an extent: the library refuses it)
        auto holds = [&](const Modes &m, const Device &t) {
            int64_t need = 1;
            for (int i = 0; i < m.n; ++i) {
                int64_t e = 0;
                for (int k = 0; k < count; ++k) if (labels[k] == m.label[i]) e = extents[k];
                if (e == 0) return false;
                if ((e - 1) > 0 && m.stride[i] > (1ll << 44) / (e - 1)) return false;
                need += (e - 1) * m.stride[i];
            }
            return need <= t.numel;
        };
        if (!holds(mA, A) || !holds(mB, B) || !holds(mC, Cout) || (a[8] != Py_None && !holds(mC, Cin))) return not_here();
        void *stream;
        if (!current_stream(a[13], stream)) return not_here();
        auto call = [&]() noexcept {
            return g_entry.contract(mA.n, mA.label, mA.stride, A.ptr, mB.n, mB.label, mB.stride, B.ptr, mC.n, mC.label, mC.stride, (const float *)Cin.ptr,
                                    (float *)Cout.ptr, count, labels, extents, alpha, beta, stream);
        };
        fg_status st;
        Py_BEGIN_ALLOW_THREADS
        st = call();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(st);
    } catch (...) {
        return not_here();
    }
}

// ---- operators on rows --------------------------------------------------------------------------------
typedef fg_status (*LayerNormFn)(int64_t, int64_t, const fg_matrix *, const void *, const void *, int32_t, float, const fg_matrix *, float *, float *, void *);
typedef fg_status (*LayerNormGradFn)(int64_t, int64_t, const fg_matrix *, const fg_matrix *, const void *, int32_t, const float *, const float *, const fg_matrix *,
                                     void *, void *, void *, int64_t, void *);
typedef fg_status (*EmbeddingFn)(int64_t, int64_t, int64_t, const fg_matrix *, const void *, int32_t, float, const fg_matrix *, void *);
typedef fg_status (*EmbeddingGradFn)(int64_t, int64_t, int64_t, const fg_matrix *, const void *, int32_t, float, const fg_matrix *, const fg_matrix *, void *, int64_t, void *);
typedef fg_status (*XentFn)(int64_t, int64_t, int64_t, const fg_matrix *, const fg_matrix *, const void *, int32_t, float, float *, float *, void *, int64_t, void *);
typedef fg_status (*XentGradFn)(int64_t, int64_t, int64_t, const fg_matrix *, const fg_matrix *, const void *, int32_t, float, const float *, const float *, int64_t,
                                const fg_matrix *, const fg_matrix *, void *, int64_t, void *);
typedef int64_t (*LayerNormSpaceFn)(int64_t, int64_t, int32_t);
typedef int64_t (*SpaceFn)(int64_t, int64_t, int64_t);
struct RowEntry {
    LayerNormFn layernorm; LayerNormGradFn layernorm_grad; LayerNormSpaceFn layernorm_grad_space;
    EmbeddingFn embedding; EmbeddingGradFn embedding_grad; SpaceFn embedding_grad_space;
    XentFn xent; SpaceFn xent_space; XentGradFn xent_grad; SpaceFn xent_grad_space;
} g_rows;

// What the binding's own marshalling checks of a call: tensors on the current GPU, of the sizes that the others have.
struct RowCall {
    int dev = -1;
    void *stream = nullptr;
    at::Tensor made;                        // a workspace from torch's allocator

    bool begin(PyObject *stream_arg) {
        PyObject *d = PyObject_CallNoArgs(g_device);
        int64_t v;
        const bool ok = as_int(d, v);
        Py_XDECREF(d);
        dev = ok ? (int)v : -1;
        return ok && current_stream(stream_arg, stream);
    }
    static int dtype_of(const at::Tensor &t) {
        switch (t.scalar_type()) {
            case at::kHalf: return FG_F16;
            case at::kBFloat16: return FG_BF16;
            case at::kFloat: return FG_F32;
            case at::kInt: return FG_I32;
            case at::kLong: return FG_I64;
            default: return -1;
        }
    }
    const at::Tensor *tensor(PyObject *o) const {
        if (!THPVariable_CheckExact(o)) return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        return t.is_cuda() && t.get_device() == dev ? &t : nullptr;
    }
    // rows, cols: -1 where they are to be read off
    bool matrix(PyObject *o, int64_t &rows, int64_t &cols, fg_matrix &m) const {
        const at::Tensor *t = tensor(o);
        if (!t || t->dim() != 2 || (rows >= 0 && t->size(0) != rows) || (cols >= 0 && t->size(1) != cols)) return false;
        rows = t->size(0);
        cols = t->size(1);
        const int dtype = dtype_of(*t);
        if ((cols > 1 && t->stride(1) != 1) || dtype < 0 || dtype > FG_F32) return false;
        m = {t->data_ptr(), nullptr, dtype, FG_ROW, rows > 1 ? t->stride(0) : t->stride(0) > cols ? t->stride(0) : cols};
        return true;
    }
    // n contiguous values of type dtype (-1: read off); absent if o is None
    bool vector(PyObject *o, int64_t n, int &dtype, void *&p) const {
        p = nullptr;
        if (o == Py_None) return true;
        const at::Tensor *t = tensor(o);
        if (!t || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1)) return false;
        const int is = dtype_of(*t);
        if (is < 0 || (dtype >= 0 && is != dtype)) return false;
        dtype = is;
        p = t->data_ptr();
        return true;
    }
    bool floats(PyObject *o, int64_t n, float *&p) const {
        int dtype = FG_F32;
        void *v;
        if (!vector(o, n, dtype, v)) return false;
        p = (float *)v;
        return true;
    }
    bool indices(PyObject *o, int64_t n, int &dtype, void *&p) const {
        dtype = -1;
        return o != Py_None && vector(o, n, dtype, p) && (dtype == FG_I32 || dtype == FG_I64);
    }
    bool workspace(PyObject *o, int64_t need, void *&p, int64_t &bytes) {
        p = nullptr;
        bytes = 0;
        if (o != Py_None) {
            const at::Tensor *t = tensor(o);
            if (!t || !t->is_contiguous()) return false;
            p = t->data_ptr();
            bytes = t->numel() * t->element_size();
        } else if (need > 0) {
            made = at::empty({need}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, (at::DeviceIndex)dev));
            p = made.data_ptr();
            bytes = need;
        }
        return true;
    }
};
template <class F> PyObject *run_rows(PyObject *const *a, Py_ssize_t n, Py_ssize_t args, F &&f) {
    if (g_forked || n != args || !g_rows.layernorm) return not_here();
    try {
        RowCall c;
        fg_status st = FG_OK;
        if (!c.begin(a[n - 1]) || !f(c, st)) return not_here();
        return PyLong_FromLong(st);
    } catch (...) {                          // no memory for a workspace, ...: the binding's own call says what is wrong
        return not_here();
    }
}
template <class F> fg_status without_gil(F &&call) {
    fg_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return st;
}

// layernorm(X, gamma, beta, eps, Y, mean, rstd, stream) -> status
PyObject *layernorm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return run_rows(a, n, 8, [&](RowCall &c, fg_status &st) {
        int64_t rows = -1, cols = -1;
        fg_matrix x, y;
        int ptype = -1;
        void *gamma, *beta;
        float eps, *mean, *rstd;
        if (!c.matrix(a[0], rows, cols, x) || !c.matrix(a[4], rows, cols, y) || !c.vector(a[1], cols, ptype, gamma) || !c.vector(a[2], cols, ptype, beta)) return false;
        if (!as_float(a[3], eps) || !c.floats(a[5], rows, mean) || !c.floats(a[6], rows, rstd)) return false;
        st = without_gil([&]() noexcept { return g_rows.layernorm(rows, cols, &x, gamma, beta, ptype < 0 ? x.dtype : ptype, eps, &y, mean, rstd, c.stream); });
        return true;
    });
}
// layernorm_grad(dY, X, gamma, mean, rstd, dX, dgamma, dbeta, workspace, stream) -> status
PyObject *layernorm_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return run_rows(a, n, 10, [&](RowCall &c, fg_status &st) {
        int64_t rows = -1, cols = -1, bytes;
        fg_matrix x, dy, dx;
        int ptype = -1;
        void *gamma, *dgamma, *dbeta, *ws;
        float *mean, *rstd;
        if (!c.matrix(a[1], rows, cols, x) || !c.matrix(a[0], rows, cols, dy) || !c.matrix(a[5], rows, cols, dx)) return false;
        if (!c.vector(a[2], cols, ptype, gamma) || !c.vector(a[6], cols, ptype, dgamma) || !c.vector(a[7], cols, ptype, dbeta)) return false;
        if (!c.floats(a[3], rows, mean) || !c.floats(a[4], rows, rstd)) return false;
        if (!c.workspace(a[8], dgamma || dbeta ? g_rows.layernorm_grad_space(rows, cols, x.dtype) : 0, ws, bytes)) return false;
        st = without_gil([&]() noexcept { return g_rows.layernorm_grad(rows, cols, &dy, &x, gamma, ptype < 0 ? x.dtype : ptype, mean, rstd, &dx, dgamma, dbeta, ws, bytes, c.stream); });
        return true;
    });
}
// embedding(table, ids, scale, Y, stream) -> status
PyObject *embedding(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return run_rows(a, n, 5, [&](RowCall &c, fg_status &st) {
        int64_t vocab = -1, dim = -1, tokens = -1;
        fg_matrix table, y;
        int kind;
        void *ids;
        float scale;
        if (!c.matrix(a[0], vocab, dim, table) || !c.matrix(a[3], tokens, dim, y) || !c.indices(a[1], tokens, kind, ids) || !as_float(a[2], scale)) return false;
        st = without_gil([&]() noexcept { return g_rows.embedding(tokens, vocab, dim, &table, ids, kind, scale, &y, c.stream); });
        return true;
    });
}
// embedding_grad(dY, ids, scale, Cin, dtable, workspace, stream) -> status
PyObject *embedding_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return run_rows(a, n, 7, [&](RowCall &c, fg_status &st) {
        int64_t vocab = -1, dim = -1, tokens = -1, bytes;
        fg_matrix dy, cin, d;
        int kind;
        void *ids, *ws;
        float scale;
        if (!c.matrix(a[4], vocab, dim, d) || !c.matrix(a[0], tokens, dim, dy) || !c.indices(a[1], tokens, kind, ids) || !as_float(a[2], scale)) return false;
        const bool add = a[3] != Py_None;
        if (add && !c.matrix(a[3], vocab, dim, cin)) return false;
        if (!c.workspace(a[5], g_rows.embedding_grad_space(tokens, vocab, dim), ws, bytes)) return false;
        st = without_gil([&]() noexcept { return g_rows.embedding_grad(tokens, vocab, dim, &dy, ids, kind, scale, add ? &cin : nullptr, &d, ws, bytes, c.stream); });
        return true;
    });
}
// xent(X, W, targets, scale, loss, lse, workspace, stream) -> status
PyObject *xent(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return run_rows(a, n, 8, [&](RowCall &c, fg_status &st) {
        int64_t vocab = -1, dim = -1, tokens = -1, bytes;
        fg_matrix x, w;
        int kind;
        void *targets, *ws;
        float scale, *loss, *lse;
        if (!c.matrix(a[0], tokens, dim, x) || !c.matrix(a[1], vocab, dim, w) || !c.indices(a[2], tokens, kind, targets) || !as_float(a[3], scale)) return false;
        if (!c.floats(a[4], tokens, loss) || !c.floats(a[5], tokens, lse) || !c.workspace(a[6], g_rows.xent_space(tokens, vocab, dim), ws, bytes)) return false;
        st = without_gil([&]() noexcept { return g_rows.xent(tokens, vocab, dim, &x, &w, targets, kind, scale, loss, lse, ws, bytes, c.stream); });
        return true;
    });
}
// xent_grad(X, W, targets, scale, lse, dloss, dX, dW, workspace, stream) -> status
PyObject *xent_grad(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return run_rows(a, n, 10, [&](RowCall &c, fg_status &st) {
        int64_t vocab = -1, dim = -1, tokens = -1, bytes;
        fg_matrix x, w, dx, dw;
        int kind;
        void *targets, *ws;
        float scale, *lse;
        if (!c.matrix(a[0], tokens, dim, x) || !c.matrix(a[1], vocab, dim, w) || !c.matrix(a[6], tokens, dim, dx) || !c.matrix(a[7], vocab, dim, dw)) return false;
        if (!c.indices(a[2], tokens, kind, targets) || !as_float(a[3], scale) || !c.floats(a[4], tokens, lse)) return false;
        const at::Tensor *g = c.tensor(a[5]);
        if (!g || g->dim() != 1 || g->size(0) != tokens || g->scalar_type() != at::kFloat) return false;
        const int64_t inc = tokens > 1 && g->stride(0) == 0 ? 0 : 1;
        if (inc && tokens > 1 && g->stride(0) != 1) return false;
        if (!c.workspace(a[8], g_rows.xent_grad_space(tokens, vocab, dim), ws, bytes)) return false;
        const float *dloss = (const float *)g->data_ptr();
        st = without_gil([&]() noexcept { return g_rows.xent_grad(tokens, vocab, dim, &x, &w, targets, kind, scale, lse, dloss, inc, &dx, &dw, ws, bytes, c.stream); });
        return true;
    });
}

// setup_rows(addresses of the entry points in the order of RowEntry)
PyObject *setup_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "setup_rows takes 10 arguments"); return nullptr; }
    void *f[10];
    for (int i = 0; i < 10; ++i) {
        f[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_rows = RowEntry{(LayerNormFn)f[0], (LayerNormGradFn)f[1], (LayerNormSpaceFn)f[2], (EmbeddingFn)f[3], (EmbeddingGradFn)f[4], (SpaceFn)f[5],
                      (XentFn)f[6], (SpaceFn)f[7], (XentGradFn)f[8], (SpaceFn)f[9]};
    Py_RETURN_NONE;
}

// setup(Matrix, raw_stream, device, addresses of fg_gemm, fg_gemm_ex, fg_gemm_noalloc, fg_gemm_dual, fg_contract)
PyObject *setup(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 8) { PyErr_SetString(PyExc_TypeError, "setup takes 8 arguments"); return nullptr; }
    void *f[5];
    for (int i = 0; i < 5; ++i) {
        f[i] = PyLong_AsVoidPtr(a[3 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_entry = Entry{(GemmFn)f[0], (GemmExFn)f[1], (GemmExFn)f[2], (DualFn)f[3], (ContractFn)f[4]};
    Py_INCREF(a[0]); Py_INCREF(a[1]); Py_INCREF(a[2]);
    g_matrix_type = a[0]; g_raw_stream = a[1]; g_device = a[2];
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {{"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, nullptr},
                           {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, nullptr},
                           {"dual", (PyCFunction)(void (*)(void))dual, METH_FASTCALL, nullptr},
                           {"contract", (PyCFunction)(void (*)(void))contract, METH_FASTCALL, nullptr},
                           {"setup_rows", (PyCFunction)(void (*)(void))setup_rows, METH_FASTCALL, nullptr},
                           {"layernorm", (PyCFunction)(void (*)(void))layernorm, METH_FASTCALL, nullptr},
                           {"layernorm_grad", (PyCFunction)(void (*)(void))layernorm_grad, METH_FASTCALL, nullptr},
                           {"embedding", (PyCFunction)(void (*)(void))embedding, METH_FASTCALL, nullptr},
                           {"embedding_grad", (PyCFunction)(void (*)(void))embedding_grad, METH_FASTCALL, nullptr},
                           {"xent", (PyCFunction)(void (*)(void))xent, METH_FASTCALL, nullptr},
                           {"xent_grad", (PyCFunction)(void (*)(void))xent_grad, METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fastcall", "Native marshalling of binding.py's calls.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
    s_re = PyUnicode_InternFromString("re");
    s_im = PyUnicode_InternFromString("im");
    s_layout = PyUnicode_InternFromString("layout");
    s_ld = PyUnicode_InternFromString("ld");
    s_dtype = PyUnicode_InternFromString("dtype");
    pthread_atfork(nullptr, nullptr, [] { g_forked = true; });
    return PyModule_Create(&g_module);
}
