// layer_call.cpp -- the short way from Python into the entry points of a layer around its attention (include/ssba.h):
// arguments checked, results allocated and the C call made in one native call, some 4 us where the interpreter and
// ctypes take 15, which is longer than most of these kernels run for a few tokens.
//
// A call that is not plainly in order (a wrong shape, type or device, no memory) returns None, and layer.py goes the long
// way, which names what is wrong. A status other than SSBA_OK comes back as a number. Nothing is kept between calls.
// The interpreter's lock is let go while results are allocated and kernels launched (cache_call.cpp has the reason).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstring>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ssba.h"

namespace {

// The library's entry points, given once by layer.py (it alone loads the library).
struct Entry {
    decltype(&ssba_rms_norm) norm;
    decltype(&ssba_rms_norm_backward) norm_backward;
    decltype(&ssba_rms_norm_backward_workspace_bytes) norm_bytes;
    decltype(&ssba_linear) linear;
    decltype(&ssba_linear_backward) linear_backward;
    decltype(&ssba_linear_backward_workspace_bytes) linear_bytes;
    decltype(&ssba_rope_axes) rope;
} g;

// A fault in a call's arguments: the long way names it.
struct Long {};

PyObject* none() { Py_RETURN_NONE; }

const at::Tensor* any(PyObject* o, int device)
{
    if (!THPVariable_Check(o)) throw Long();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device) throw Long();
    return &t;
}

const at::Tensor* dense(PyObject* o, int device, at::ScalarType type)
{
    const at::Tensor* t = any(o, device);
    if (t->scalar_type() != type || !t->is_contiguous()) throw Long();
    return t;
}

const at::Tensor* matrix(PyObject* o, int device, at::ScalarType type, int64_t rows, int64_t cols)
{
    const at::Tensor* t = dense(o, device, type);
    if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) throw Long();
    return t;
}

const at::Tensor* vector(PyObject* o, int device, int64_t n)
{
    const at::Tensor* t = dense(o, device, at::kFloat);
    if (t->dim() != 1 || t->size(0) != n) throw Long();
    return t;
}

const void* data(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }
const float* floats(const at::Tensor* t) { return t ? t->const_data_ptr<float>() : nullptr; }
void* out(at::Tensor& t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
float* out_floats(at::Tensor& t) { return t.defined() ? t.mutable_data_ptr<float>() : nullptr; }

at::Tensor make(int device, at::IntArrayRef size, at::ScalarType type)
{
    return at::empty(size, at::TensorOptions().dtype(type).device(c10::Device(c10::kCUDA, device)));
}

int here() { return c10::cuda::current_device(); }

void* stream(int device) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream(); }

int32_t narrow(int64_t n)
{
    if (n > INT32_MAX) throw Long();
    return (int32_t)n;
}

long number(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Long();
    }
    return v;
}

bool truth(PyObject* o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) {
        PyErr_Clear();
        throw Long();
    }
    return v != 0;
}

double real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Long();
    }
    return v;
}

struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    Unlocked& operator=(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

PyObject* wrap(at::Tensor& t) { return t.defined() ? THPVariable_Wrap(std::move(t)) : none(); }

PyObject* held(PyObject* o)
{
    Py_INCREF(o);
    return o;
}

// Runs a call's body; what is not plainly in order, or throws, is None.
template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F&& f)
{
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return f();
    } catch (...) {
        return none();
    }
}

// (addresses of the entry points, in the order of Entry)
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long f[7];
    if (!PyArg_ParseTuple(args, "KKKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6])) return nullptr;
    static_assert(sizeof(Entry) == sizeof(f), "seven addresses");
    std::memcpy(&g, f, sizeof(g));
    return none();
}

at::ScalarType norm_type(const at::Tensor* t)
{
    if (t->scalar_type() != at::kBFloat16 && t->scalar_type() != at::kFloat) throw Long();
    return t->scalar_type();
}

// (x, w, residual or None, eps, e4m3) -> (y, h, rstd) or (y, scale, h, rstd)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 5, [&]() -> PyObject* {
        const int dev = here();
        const at::Tensor* x = any(a[0], dev);
        const at::ScalarType type = norm_type(x);
        if (x->dim() != 2 || !x->is_contiguous()) throw Long();
        const int32_t T = narrow(x->size(0)), D = narrow(x->size(1));
        const at::Tensor *w = vector(a[1], dev, D), *r = a[2] == Py_None ? nullptr : matrix(a[2], dev, type, T, D);
        const float eps = (float)real(a[3]);
        const bool e4m3 = truth(a[4]);
        at::Tensor y, h, scale, rstd;
        int rc;
        {
            Unlocked scope;
            y = make(dev, {T, D}, e4m3 ? at::kFloat8_e4m3fn : type);
            if (r) h = make(dev, {T, D}, type);
            if (e4m3) scale = make(dev, {T}, at::kFloat);
            rstd = make(dev, {T}, at::kFloat);
            rc = g.norm(data(x), data(r), floats(w), T, D, type == at::kFloat ? SSBA_FP32 : SSBA_BF16, eps, out(h), out(y),
                        out_floats(scale), out_floats(rstd), stream(dev));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        PyObject* hh = r ? wrap(h) : held(a[0]);
        return e4m3 ? Py_BuildValue("NNNN", wrap(y), wrap(scale), hh, wrap(rstd)) : Py_BuildValue("NNN", wrap(y), hh, wrap(rstd));
    });
}

// (dy, h, w, rstd, dh or None) -> (dx, dw)
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 5, [&]() -> PyObject* {
        const int dev = here();
        const at::Tensor* h = any(a[1], dev);
        const at::ScalarType type = norm_type(h);
        if (h->dim() != 2 || !h->is_contiguous()) throw Long();
        const int32_t T = narrow(h->size(0)), D = narrow(h->size(1)), code = type == at::kFloat ? SSBA_FP32 : SSBA_BF16;
        const at::Tensor *dy = matrix(a[0], dev, type, T, D), *w = vector(a[2], dev, D), *rstd = vector(a[3], dev, T);
        const at::Tensor* dh = a[4] == Py_None ? nullptr : matrix(a[4], dev, type, T, D);
        at::Tensor dx, dw, ws;
        int rc;
        {
            Unlocked scope;
            const size_t need = g.norm_bytes(T, D, code);
            dx = make(dev, {T, D}, type);
            dw = make(dev, {D}, at::kFloat);
            ws = make(dev, {(int64_t)need}, at::kByte);
            rc = g.norm_backward(data(dy), data(h), floats(w), floats(rstd), data(dh), T, D, code, out(dx), out_floats(dw), out(ws),
                                 need, stream(dev));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        return Py_BuildValue("NN", wrap(dx), wrap(dw));
    });
}

// (x, W, bias, residual, x_scale, w_scale (each or None), act, pre, gated) -> y or (y, z)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 9, [&]() -> PyObject* {
        const int dev = here();
        const at::Tensor* x = any(a[0], dev);
        const at::ScalarType type = x->scalar_type();
        const bool f8 = type == at::kFloat8_e4m3fn, pre = truth(a[7]), gated = truth(a[8]);
        if ((!f8 && type != at::kBFloat16) || x->dim() != 2 || !x->is_contiguous()) throw Long();
        const at::Tensor* W = dense(a[1], dev, type);
        if (W->dim() != 2 || W->size(1) != x->size(1) || (gated && W->size(0) % 2)) throw Long();
        const int32_t T = narrow(x->size(0)), K = narrow(x->size(1)), rows = narrow(W->size(0)), N = gated ? rows / 2 : rows;
        const at::Tensor *bias = a[2] == Py_None ? nullptr : vector(a[2], dev, N);
        const at::Tensor *r = a[3] == Py_None ? nullptr : matrix(a[3], dev, at::kBFloat16, T, N);
        const at::Tensor *xs = a[4] == Py_None ? nullptr : vector(a[4], dev, T), *ws = a[5] == Py_None ? nullptr : vector(a[5], dev, rows);
        const ssba_linear_desc d{T, N, K, f8 ? SSBA_E4M3 : SSBA_BF16, (int32_t)number(a[6]), gated};
        at::Tensor y, z;
        int rc;
        {
            Unlocked scope;
            y = make(dev, {T, N}, at::kBFloat16);
            if (pre) z = make(dev, {T, rows}, at::kBFloat16);
            rc = g.linear(&d, data(x), data(W), floats(xs), floats(ws), floats(bias), data(r), out(y), out(z), stream(dev));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        return pre ? Py_BuildValue("NN", wrap(y), wrap(z)) : wrap(y);
    });
}

// (dy, x or None, W or None, z or None, act, gated, bias, whether dx and dW are wanted) -> (dx, dW, db, each or None)
PyObject* linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 9, [&]() -> PyObject* {
        const int dev = here();
        const at::Tensor* dy = dense(a[0], dev, at::kBFloat16);
        const bool gated = truth(a[5]), bias = truth(a[6]), want_dx = truth(a[7]), want_dW = truth(a[8]);
        if (dy->dim() != 2 || (!want_dx && !want_dW)) throw Long();
        const int32_t T = narrow(dy->size(0)), N = narrow(dy->size(1)), rows = narrow((int64_t)N * (gated ? 2 : 1));
        const at::Tensor* one = dense(want_dx ? a[2] : a[1], dev, at::kBFloat16);
        if (one->dim() != 2) throw Long();
        const int32_t K = narrow(one->size(1));
        const at::Tensor* W = want_dx ? matrix(a[2], dev, at::kBFloat16, rows, K) : nullptr;
        const at::Tensor* x = want_dW ? matrix(a[1], dev, at::kBFloat16, T, K) : nullptr;
        const int32_t act = (int32_t)number(a[4]);
        if ((act != 0) != (a[3] != Py_None)) throw Long();
        const at::Tensor* z = act ? matrix(a[3], dev, at::kBFloat16, T, rows) : nullptr;
        const ssba_linear_desc d{T, N, K, SSBA_BF16, act, gated};
        at::Tensor dx, dW, db, ws;
        int rc;
        {
            Unlocked scope;
            const size_t need = g.linear_bytes(&d);
            if (want_dx) dx = make(dev, {T, K}, at::kBFloat16);
            if (want_dW) dW = make(dev, {rows, K}, at::kBFloat16);
            if (bias) db = make(dev, {N}, at::kFloat);
            if (need) ws = make(dev, {(int64_t)need}, at::kByte);
            rc = g.linear_backward(&d, data(dy), data(x), data(W), data(z), out(dx), out(dW), out_floats(db), out(ws), need, stream(dev));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        PyObject *p = wrap(dx), *q = wrap(dW);
        return Py_BuildValue("NNN", p, q, wrap(db));
    });
}

// A head tensor's four sizes and three strides; false without a last dimension side by side.
bool heads(const at::Tensor* t, int64_t* size, int64_t* stride)
{
    const int64_t k = t->dim();
    if ((k != 3 && k != 4) || (t->size(k - 1) != 1 && t->stride(k - 1) != 1)) return false;
    size[0] = 1;
    stride[0] = 0;
    for (int64_t i = 0; i < k; ++i) {
        size[4 - k + i] = t->size(i);
        if (i < k - 1) stride[4 - k + i] = t->stride(i);
    }
    return true;
}

// Whether no two elements share an address: by stride, each dimension steps past those inside it.
bool apart(const int64_t* size, const int64_t* stride)
{
    int64_t s[4] = {stride[0], stride[1], stride[2], 1};
    int order[4] = {3, 2, 1, 0};
    for (int i = 1; i < 4; ++i)
        for (int j = i; j > 0 && s[order[j]] < s[order[j - 1]]; --j) std::swap(order[j], order[j - 1]);
    int64_t reach = 1;
    for (int i : order) {
        if (size[i] <= 1) continue;
        if (s[i] < reach) return false;
        reach += s[i] * (size[i] - 1);
    }
    return true;
}

// (x, positions, axes, base, layout, shared, inverse, out or None) -> out
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded(n, 8, [&]() -> PyObject* {
        const int dev = here();
        const at::Tensor *x = any(a[0], dev), *pos = dense(a[1], dev, at::kInt);
        const at::ScalarType type = norm_type(x);
        int64_t size[4], xs[3], osize[4], os[3];
        if (!heads(x, size, xs) || !PyTuple_Check(a[2])) throw Long();
        const Py_ssize_t A = PyTuple_GET_SIZE(a[2]);
        if (A < 1 || A > SSBA_ROPE_MAX_AXES) throw Long();
        ssba_rope_desc d = {};
        d.B = narrow(size[0]);
        d.T = narrow(size[1]);
        d.heads = narrow(size[2]);
        d.head_dim = narrow(size[3]);
        d.axes = (int32_t)A;
        for (Py_ssize_t i = 0; i < A; ++i) {
            const long v = number(PyTuple_GET_ITEM(a[2], i));
            if (v <= 0 || v > 65535) throw Long();
            d.sections[i] = (int32_t)v;
        }
        d.base = real(a[3]);
        d.layout = (int32_t)number(a[4]);
        d.shared = truth(a[5]);
        d.inverse = truth(a[6]);
        d.dtype = type == at::kFloat ? SSBA_FP32 : SSBA_BF16;
        const int64_t k = pos->dim();
        if ((k != 2 && k != 3) || pos->size(k - 1) != A || pos->size(k - 2) != size[1] || (k == 3 && pos->size(0) != size[0])) throw Long();
        at::Tensor made;
        const at::Tensor* o = nullptr;
        if (a[7] != Py_None) {
            o = any(a[7], dev);
            if (o->scalar_type() != type || o->dim() != x->dim() || !heads(o, osize, os) || std::memcmp(size, osize, sizeof(size)) ||
                !apart(osize, os))
                throw Long();
        }
        int rc;
        {
            Unlocked scope;
            if (!o) {
                made = make(dev, x->sizes(), type);
                heads(&made, osize, os);
            }
            rc = g.rope(&d, x->const_data_ptr(), xs, pos->const_data_ptr<int32_t>(), k == 3 ? size[1] * A : 0,
                        o ? o->mutable_data_ptr() : made.mutable_data_ptr(), os, stream(dev));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        return o ? held(a[7]) : wrap(made);
    });
}

template <class F>
PyCFunction fast(F f)
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef kMethods[] = {{"bind", bind, METH_VARARGS, nullptr},
                          {"rms_norm", fast(rms_norm), METH_FASTCALL, nullptr},
                          {"rms_norm_backward", fast(rms_norm_backward), METH_FASTCALL, nullptr},
                          {"linear", fast(linear), METH_FASTCALL, nullptr},
                          {"linear_backward", fast(linear_backward), METH_FASTCALL, nullptr},
                          {"rope", fast(rope), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_layer_call", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_call(void) { return PyModule_Create(&kModule); }
