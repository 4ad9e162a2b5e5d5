// cache_call.cpp -- the short way from Python into the cache's entry points (include/ssba.h): arguments checked, results
// allocated and the C call made in one native call, 3 to 5 us where the interpreter and ctypes take 15. A serving step
// makes such a call several times a layer, and most of them run for less than that on the GPU.
//
// A call that is not plainly in order (a wrong shape, type or device, results that are not to be allocated on the
// current stream, no memory) returns None, and cache.py goes the long way, which names what is wrong. A status other than SSBA_OK comes
// back as a number. Nothing is kept between calls.
//
// The interpreter's lock is held while arguments are looked at, and not while results are allocated or kernels launched: either
// may wait for the GPU, and what the GPU waits for (a host callback, another thread's copy) may need the lock. The caller's
// references keep the arguments' tensors meanwhile.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ssba.h"

namespace {

typedef decltype(&ssba_cache_append) AppendFn;
typedef decltype(&ssba_cache_select) SelectFn;
typedef decltype(&ssba_cache_attend) AttendFn;
typedef decltype(&ssba_cache_copy) CopyFn;

// What calls with one descriptor on one pool have in common. The descriptor and the pool are copies; the pool's tensors
// are kept alive by the Cache that holds this.
struct Call {
    AppendFn append;
    SelectFn select;
    AttendFn attend;
    CopyFn copy;
    ssba_cache_desc desc;
    ssba_cache pool;
    int device;
    at::ScalarType type;
};

const char kName[] = "ssba.cache_call";

void drop(PyObject* capsule) { delete static_cast<Call*>(PyCapsule_GetPointer(capsule, kName)); }

const at::Tensor* tensor(PyObject* o, const Call& c, at::ScalarType type)
{
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != c.device || t.scalar_type() != type || !t.is_contiguous()) return nullptr;
    return &t;
}

struct Batch {
    const int32_t *table, *lens, *cu;
    int32_t width, B;
};

bool batch(PyObject* const* a, const Call& c, Batch& b)
{
    const at::Tensor *t = tensor(a[0], c, at::kInt), *l = tensor(a[1], c, at::kInt), *u = tensor(a[2], c, at::kInt);
    if (!t || !l || !u || t->dim() != 2 || l->dim() != 1 || u->dim() != 1 || t->size(0) > INT32_MAX - 1 ||
        t->size(1) > INT32_MAX || l->size(0) != t->size(0) || u->size(0) != t->size(0) + 1)
        return false;
    b = Batch{t->const_data_ptr<int32_t>(), l->const_data_ptr<int32_t>(), u->const_data_ptr<int32_t>(), (int32_t)t->size(1),
              (int32_t)t->size(0)};
    return true;
}

// [T, heads, head_dim] of the call's type.
const at::Tensor* rows(PyObject* o, const Call& c, int heads)
{
    const at::Tensor* t = tensor(o, c, c.type);
    if (!t || t->dim() != 3 || t->size(0) > INT32_MAX || t->size(1) != heads || t->size(2) != c.desc.head_dim) return nullptr;
    return t;
}

at::Tensor make(const Call& c, at::IntArrayRef size, at::ScalarType type)
{
    return at::empty(size, at::TensorOptions().dtype(type).device(c10::Device(c10::kCUDA, c.device)));
}

PyObject* none() { Py_RETURN_NONE; }

const Call* call_of(PyObject* const* a, Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    return static_cast<Call*>(PyCapsule_GetPointer(a[0], kName));
}

// Without the interpreter's lock, to the end of the scope (also by an exception).
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    Unlocked& operator=(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

bool elsewhere(const Call& c) { return c10::cuda::current_device() != c.device; }

void* stream(const Call& c) { return c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(c.device)).stream(); }

// (addresses of append, select, attend, copy, descriptor and pool; device; bf16) -> what the others take first
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long f[6];
    int device, bf16;
    if (!PyArg_ParseTuple(args, "KKKKKKip", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &device, &bf16)) return nullptr;
    Call* c = new (std::nothrow) Call;
    if (!c) return PyErr_NoMemory();
    c->append = reinterpret_cast<AppendFn>(f[0]);
    c->select = reinterpret_cast<SelectFn>(f[1]);
    c->attend = reinterpret_cast<AttendFn>(f[2]);
    c->copy = reinterpret_cast<CopyFn>(f[3]);
    c->desc = *reinterpret_cast<const ssba_cache_desc*>(f[4]);
    c->pool = *reinterpret_cast<const ssba_cache*>(f[5]);
    c->device = device;
    c->type = bf16 ? at::kBFloat16 : at::kFloat;
    return PyCapsule_New(c, kName, drop);
}

// (call, k, v, table, lens, cu)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    const Call* c = call_of(a, n, 6);
    if (!c) return nullptr;
    try {
        Batch b;
        const at::Tensor *k = rows(a[1], *c, c->desc.kv_heads), *v = rows(a[2], *c, c->desc.kv_heads);
        if (elsewhere(*c) || !k || !v || v->size(0) != k->size(0) || !batch(a + 3, *c, b)) return none();
        int rc;
        {
            Unlocked scope;
            rc = c->append(&c->desc, &c->pool, k->const_data_ptr(), v->const_data_ptr(), (int32_t)k->size(0), b.table, b.width,
                           b.lens, b.cu, b.B, stream(*c));
        }
        return PyLong_FromLong(rc);
    } catch (...) {
        return none();
    }
}

// (call, q, table, lens, cu, keep, first) -> (idx, cnt)
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    const Call* c = call_of(a, n, 7);
    if (!c) return nullptr;
    const long keep = PyLong_AsLong(a[5]), first = PyLong_AsLong(a[6]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return none();
    }
    try {
        Batch b;
        const at::Tensor* q = rows(a[1], *c, c->desc.heads);
        if (elsewhere(*c) || !q || !batch(a + 2, *c, b) || first < 0 || keep <= first || keep > SSBA_CACHE_MAX_WIDTH)
            return none();
        at::Tensor idx, cnt;
        int rc;
        {
            Unlocked scope;
            idx = make(*c, {q->size(0), c->desc.kv_heads, keep}, at::kInt);
            cnt = make(*c, {q->size(0), c->desc.kv_heads}, at::kInt);
            rc = c->select(&c->desc, &c->pool, q->const_data_ptr(), (int32_t)q->size(0), b.table, b.width, b.lens, b.cu, b.B,
                           (int32_t)keep, (int32_t)first, idx.mutable_data_ptr<int32_t>(), cnt.mutable_data_ptr<int32_t>(),
                           stream(*c));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        PyObject *x = THPVariable_Wrap(std::move(idx)), *y = THPVariable_Wrap(std::move(cnt));
        return Py_BuildValue("NN", x, y);
    } catch (...) {
        return none();
    }
}

// (call, q, table, lens, cu, idx or None, cnt or None, workspace) -> (O, lse)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    const Call* c = call_of(a, n, 8);
    if (!c) return nullptr;
    try {
        Batch b;
        const at::Tensor *q = rows(a[1], *c, c->desc.heads), *ws = tensor(a[7], *c, at::kByte);
        if (elsewhere(*c) || !q || !ws || !batch(a + 2, *c, b)) return none();
        const at::Tensor *idx = nullptr, *cnt = nullptr;
        if (a[5] != Py_None || a[6] != Py_None) {
            idx = tensor(a[5], *c, at::kInt);
            cnt = tensor(a[6], *c, at::kInt);
            if (!idx || !cnt || idx->dim() != 3 || cnt->dim() != 2 || idx->size(0) != q->size(0) || cnt->size(0) != q->size(0) ||
                idx->size(1) != c->desc.kv_heads || cnt->size(1) != c->desc.kv_heads || idx->size(2) > SSBA_CACHE_MAX_WIDTH)
                return none();
        }
        at::Tensor O, lse;
        int rc;
        {
            Unlocked scope;
            O = make(*c, q->sizes(), c->type);
            lse = make(*c, {q->size(0), q->size(1)}, at::kFloat);
            rc = c->attend(&c->desc, &c->pool, q->const_data_ptr(), (int32_t)q->size(0), b.table, b.width, b.lens, b.cu, b.B,
                           idx ? idx->const_data_ptr<int32_t>() : nullptr, cnt ? cnt->const_data_ptr<int32_t>() : nullptr,
                           idx ? (int32_t)idx->size(2) : 0, O.mutable_data_ptr(), lse.mutable_data_ptr<float>(),
                           ws->mutable_data_ptr(), (size_t)ws->numel(), stream(*c));
        }
        if (rc != SSBA_OK) return PyLong_FromLong(rc);
        PyObject *x = THPVariable_Wrap(std::move(O)), *y = THPVariable_Wrap(std::move(lse));
        return Py_BuildValue("NN", x, y);
    } catch (...) {
        return none();
    }
}

// (call, src, dst)
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    const Call* c = call_of(a, n, 3);
    if (!c) return nullptr;
    try {
        const at::Tensor *s = tensor(a[1], *c, at::kInt), *d = tensor(a[2], *c, at::kInt);
        if (elsewhere(*c) || !s || !d || s->dim() != 1 || d->dim() != 1 || s->size(0) != d->size(0) || s->size(0) > INT32_MAX)
            return none();
        int rc;
        {
            Unlocked scope;
            rc = c->copy(&c->desc, &c->pool, s->const_data_ptr<int32_t>(), d->const_data_ptr<int32_t>(), (int32_t)s->size(0),
                         stream(*c));
        }
        return PyLong_FromLong(rc);
    } catch (...) {
        return none();
    }
}

template <class F>
PyCFunction fast(F f)
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef kMethods[] = {{"bind", bind, METH_VARARGS, nullptr},
                          {"append", fast(append), METH_FASTCALL, nullptr},
                          {"select", fast(select), METH_FASTCALL, nullptr},
                          {"attend", fast(attend), METH_FASTCALL, nullptr},
                          {"copy", fast(copy), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_cache_call", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cache_call(void) { return PyModule_Create(&kModule); }
