// Python calls of the batch-serving operators straight from torch tensors: checks of the arguments and marshalling only, the work is
// libaq's (include/aq.h).  A decode step makes three of these calls per layer; through ctypes one cost the host 6.3 to 9.5 us (here 2.6 to
// 3.5), most of it in asking tensors for their properties from Python and in converting up to fifteen arguments.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/aq.h"

namespace {

decltype(&aq_kv8_plan) g_plan;
decltype(&aq_kv8_append) g_append;
decltype(&aq_kv8_attn) g_attn;
decltype(&aq_rope_rows) g_rope;

struct Refused {};   // a Python error is set

[[noreturn]] void refuse(const char* what, const char* why) {
    PyErr_Format(PyExc_ValueError, "%s: %s", what, why);
    throw Refused{};
}

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) refuse(what, "a torch tensor is wanted");
    return THPVariable_Unpack(o);
}

void here(const at::Tensor& t, int dev, const char* what) {
    if (!t.is_cuda() || t.get_device() != dev) {
        PyErr_Format(PyExc_ValueError, "%s: a tensor on %s, and the current device is cuda:%d", what, t.device().str().c_str(), dev);
        throw Refused{};
    }
}

// Address of a contiguous int32 array.
int32_t* ints(PyObject* o, int dev, const char* what, int64_t want = -1) {
    const at::Tensor& t = tensor(o, what);
    here(t, dev, what);
    if (t.scalar_type() != at::kInt || !t.is_contiguous()) refuse(what, "a contiguous tensor of int32 is wanted");
    if (want >= 0 && t.numel() != want) refuse(what, "not as long as the step's other arrays ask for");
    return static_cast<int32_t*>(t.data_ptr());
}

int type_of(const at::Tensor& t, const char* what) {
    switch (t.scalar_type()) {
        case at::kHalf: return AQ_F16;
        case at::kBFloat16: return AQ_BF16;
        case at::kFloat: return AQ_F32;
        default: refuse(what, "float16, bfloat16 or float32 is wanted");
    }
}

// Rows [n_rows][heads][head_dim]: rows may be apart, a row's heads lie together.
struct Rows {
    void* p;
    int64_t n, heads, dim, stride;
    aq_dtype_t type;
};
Rows rows(PyObject* o, int dev, const char* what) {
    const at::Tensor& t = tensor(o, what);
    here(t, dev, what);
    if (t.dim() != 3) refuse(what, "rows [n_rows][heads][head_dim] are wanted");
    const auto size = t.sizes(), stride = t.strides();
    if ((stride[2] != 1 && size[2] > 1) || (stride[1] != size[2] && size[1] > 1)) refuse(what, "the heads of a row have to lie together");
    return Rows{t.data_ptr(), size[0], size[1], size[2], size[0] > 1 ? stride[0] : size[1] * size[2], (aq_dtype_t)type_of(t, what)};
}

long long number(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
}

aq_stream_t stream(PyObject* o, int dev) {   // a stream's handle, or None: torch's current one
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
    return reinterpret_cast<aq_stream_t>(static_cast<intptr_t>(number(o)));
}

// cache or step: (address, device) as the descriptors hold them
template <typename T>
const T* descriptor(PyObject* addr, PyObject* device, int dev, const char* what) {
    if (number(device) != dev) refuse(what, "on another device than the current one");
    return reinterpret_cast<const T*>(static_cast<intptr_t>(number(addr)));
}

template <typename Fn>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, Fn fn) {
    if (n != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong((long)fn(c10::cuda::current_device()));
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// lens, new, table, free, n_free, page, lens_out, n_free_out, row_start, pos, stream
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&](int dev) {
        const at::Tensor& table = tensor(a[2], "table");
        if (table.dim() != 2) refuse("table", "[n_seqs][width] is wanted");
        const int64_t seqs = table.size(0), width = table.size(1);
        if (seqs > AQ_KV8_MAX_SEQS) return AQ_ERR_UNSUPPORTED;
        return g_plan(ints(a[0], dev, "lens", seqs), ints(a[1], dev, "new", seqs), (int)seqs, (int)number(a[5]), ints(a[2], dev, "table"), width,
                      ints(a[3], dev, "free"), tensor(a[3], "free").numel(), ints(a[4], dev, "n_free", 1), ints(a[6], dev, "lens_out", seqs),
                      ints(a[7], dev, "n_free_out", 1), ints(a[8], dev, "row_start", seqs + 1), ints(a[9], dev, "pos"),
                      tensor(a[9], "pos").numel(), stream(a[10], dev));
    });
}

// cache, its device, step, its device, k, v, stream
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&](int dev) {
        const auto* c = descriptor<aq_kv8_cache_t>(a[0], a[1], dev, "cache");
        const auto* b = descriptor<aq_kv8_batch_t>(a[2], a[3], dev, "batch");
        const Rows k = rows(a[4], dev, "k"), v = rows(a[5], dev, "v");
        if (k.n != v.n || k.heads != v.heads || k.dim != v.dim || k.stride != v.stride || k.type != v.type || k.heads != c->n_kv_heads || k.dim != c->head_dim)
            refuse("k, v", "rows of the cache's heads, of one type and stride, are wanted");
        return g_append(c, b, k.p, v.p, k.stride, k.n, k.type, stream(a[6], dev));
    });
}

// cache, its device, step, its device, q, out, scratch, scale, stream
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&](int dev) {
        const auto* c = descriptor<aq_kv8_cache_t>(a[0], a[1], dev, "cache");
        const auto* b = descriptor<aq_kv8_batch_t>(a[2], a[3], dev, "batch");
        const Rows q = rows(a[4], dev, "q"), o = rows(a[5], dev, "out");
        if (q.n != o.n || q.heads != o.heads || q.dim != o.dim || q.dim != c->head_dim || q.heads > INT32_MAX)
            refuse("q, out", "rows of heads alike, of the cache's dimension, are wanted");
        const at::Tensor& s = tensor(a[6], "scratch");
        here(s, dev, "scratch");
        if (!s.is_contiguous()) refuse("scratch", "a contiguous tensor is wanted");
        const double scale = PyFloat_AsDouble(a[7]);
        if (scale == -1.0 && PyErr_Occurred()) throw Refused{};
        return g_attn(c, b, q.p, q.stride, o.p, o.stride, q.n, (int)q.heads, (float)scale, q.type, o.type, s.data_ptr(), s.nbytes(), stream(a[8], dev));
    });
}

// frequencies, x, pos, out, stream
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&](int dev) {
        const auto* r = reinterpret_cast<const aq_rope_t*>(static_cast<intptr_t>(number(a[0])));
        const Rows x = rows(a[1], dev, "x"), o = rows(a[3], dev, "out");
        if (x.n != o.n || x.heads != o.heads || x.dim != o.dim) refuse("x, out", "rows of heads alike are wanted");
        if (x.heads > 4096 || x.dim > 1024) return AQ_ERR_UNSUPPORTED;
        return g_rope(r, x.p, x.type, x.stride, o.p, o.type, o.stride, x.n, (int)x.heads, (int)x.dim, ints(a[2], dev, "pos", x.n), stream(a[4], dev));
    });
}

// addresses of aq_kv8_plan, aq_kv8_append, aq_kv8_attn, aq_rope_rows in the loaded library
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "four addresses are wanted");
        return nullptr;
    }
    g_plan = reinterpret_cast<decltype(g_plan)>(PyLong_AsVoidPtr(a[0]));
    g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[1]));
    g_attn = reinterpret_cast<decltype(g_attn)>(PyLong_AsVoidPtr(a[2]));
    g_rope = reinterpret_cast<decltype(g_rope)>(PyLong_AsVoidPtr(a[3]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

#define AQ_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL
PyMethodDef methods[] = {{"bind", AQ_FAST(bind), nullptr},     {"plan", AQ_FAST(plan), nullptr}, {"append", AQ_FAST(append), nullptr},
                         {"attn", AQ_FAST(attn), nullptr},     {"rope", AQ_FAST(rope), nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_aq_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__aq_torch() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", AQ_BUILT_FOR) < 0) {   // the interpreter and the torch that it was compiled against
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
