// The calls of the paged cache from Python, without what they cost there: a decode step makes five of them, each of 2.4 us for its launch, and a
// check of one tensor's type, shape and place takes 0.4 us in Python (20 ns here), the conversions of twelve arguments by ctypes 2.
// Arguments are checked against the structs of include/gsa.h, then the library's function is called at the address that bind() was given.
//
// call(address, a, b, ...) calls any function of the library that takes up to sixteen integers or pointers and returns an int, with the
// given ints (None: NULL).  In the x86-64 and AArch64 calling conventions a narrower integer argument occupies a whole register or stack
// slot, so that all of them can be passed as 64 bits.  The binding's calls go by the functions further down, which check their arguments; this one
// checks nothing and serves the test of the calling convention.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <exception>
#include <string>
#include <vector>

#include "gsa.h"

namespace {

constexpr Py_ssize_t kMost = 16;
typedef int (*fn_t)(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t,
                    int64_t, int64_t, int64_t);

PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    int64_t v[kMost + 1] = {0};
    if (n < 1 || n > kMost + 1) {
        PyErr_SetString(PyExc_TypeError, "call(address, up to 16 integers)");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (args[i] == Py_None) continue;
        if (!PyLong_Check(args[i])) {
            PyErr_SetString(PyExc_TypeError, "arguments are ints or None");
            return nullptr;
        }
        // (addresses and sizes are unsigned, lengths signed: the low 64 bits are right for either)
        v[i] = (int64_t)PyLong_AsUnsignedLongLongMask(args[i]);
        if (v[i] == -1 && PyErr_Occurred()) return nullptr;
    }
    if (!v[0]) {
        PyErr_SetString(PyExc_ValueError, "no function");
        return nullptr;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((fn_t)(intptr_t)v[0])(v[1], v[2], v[3], v[4], v[5], v[6], v[7], v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15], v[16]);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// ---- the cache's calls -----------------------------------------------------------------------------------------------------
PyObject* g_error = nullptr;                               // GsaError
struct {
    decltype(&gsa_cache_reserve) reserve;
    decltype(&gsa_cache_append) append;
    decltype(&gsa_cache_read) read;
    decltype(&gsa_cache_fork) fork;
    decltype(&gsa_cache_release) release;
    decltype(&gsa_cache_compact) compact;
    decltype(&gsa_cache_indexer_scores) indexer_scores;
    decltype(&gsa_cache_topk) topk;
    decltype(&gsa_cache_attn_fwd) attn_fwd;
} g_fn = {};

struct Refused : std::exception {                          // an argument that does not fit
    std::string what_;
    explicit Refused(std::string s) : what_(std::move(s)) {}
    const char* what() const noexcept override { return what_.c_str(); }
};

constexpr at::ScalarType kBf16 = at::ScalarType::BFloat16, kF32 = at::ScalarType::Float, kI32 = at::ScalarType::Int;

// a call's arguments: cache, device, ... , workspace, stream
struct Args {
    PyObject* const* a;
    const gsa_cache_t* c;
    int device;
    void *ws, *stream;
    size_t ws_bytes;

    static int64_t integer(PyObject* o) {
        if (!PyLong_Check(o)) throw Refused("expected an int");
        const int64_t v = (int64_t)PyLong_AsUnsignedLongLongMask(o);
        if (v == -1 && PyErr_Occurred()) PyErr_Clear();
        return v;
    }
    const at::Tensor* tensor(int i) const {
        if (a[i] == Py_None) return nullptr;
        if (!THPVariable_Check(a[i])) throw Refused(std::string("expected a tensor, got ") + Py_TYPE(a[i])->tp_name);
        return &THPVariable_Unpack(a[i]);
    }
    Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : a(args) {
        if (n != want) throw Refused("a wrong number of arguments");
        if (!g_error) throw Refused("bind() first");
        c = (const gsa_cache_t*)(intptr_t)integer(a[0]);
        device = (int)integer(a[1]);
        const at::Tensor* w = tensor((int)n - 2);
        if (!c || !w || !w->is_cuda() || w->get_device() != device || !w->is_contiguous() || c10::cuda::current_device() != device)
            throw Refused("the cache, a contiguous workspace and the current device belong together");
        ws = w->mutable_data_ptr();
        ws_bytes = w->nbytes();
        stream = a[n - 1] == Py_None ? (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream() : (void*)(intptr_t)integer(a[n - 1]);
    }
    // address of argument i, a contiguous tensor of that type and shape on the cache's device; NULL for None
    void* at(int i, at::ScalarType type, std::initializer_list<int64_t> shape) const {
        const at::Tensor* t = tensor(i);
        if (!t) return nullptr;
        if (t->scalar_type() == type && t->sizes() == at::IntArrayRef(shape) && t->is_cuda() && t->get_device() == device && t->is_contiguous())
            return t->mutable_data_ptr();
        auto sizes = [](at::IntArrayRef s) {
            std::string r = "(";
            for (int64_t x : s) r += (r.size() > 1 ? ", " : "") + std::to_string(x);
            return r + ")";
        };
        throw Refused(std::string("expected a contiguous ") + c10::toString(type) + " tensor " + sizes(shape) + " on GPU " + std::to_string(device) + ", got " +
                      c10::toString(t->scalar_type()) + " " + sizes(t->sizes()) + " on " + t->device().str());
    }
    // rows a sequence of argument i, [B, L, ...]
    int64_t rows(int i, const char* none) const {
        const at::Tensor* t = tensor(i);
        if (!t || t->dim() < 2) throw Refused(none);
        if (t->size(1) > INT32_MAX) throw Refused("too many rows");
        return t->size(1);
    }
    const gsa_params_t* params(int i) const {
        const gsa_params_t* p = (const gsa_params_t*)(intptr_t)integer(a[i]);
        if (!p) throw Refused("no parameters");
        return p;
    }
};

// runs f(args) -> gsa_status, without the interpreter's lock once the arguments are known
template <class F>
PyObject* guarded(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F f) {
    try {
        const Args k(a, n, want);
        return PyLong_FromLong(f(k));
    } catch (const std::exception& e) {
        PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}
template <class F>
int unlocked(F f) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// (c, device, n_new, start, ws, stream)
PyObject* reserve(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 6, [](const Args& k) {
        const auto* n_new = (const int32_t*)k.at(2, kI32, {k.c->B});
        auto* start = (int32_t*)k.at(3, kI32, {k.c->B});
        return unlocked([&] { return g_fn.reserve(k.c, n_new, start, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, K, V, g2, kI, n_new, start, ws, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 10, [](const Args& k) {
        const int64_t B = k.c->B, L = k.rows(5, "kI is [B, L_new, dI]");
        const std::initializer_list<int64_t> kv = {B, L, k.c->n_kv, k.c->d_h};
        const void *K = k.at(2, kBf16, kv), *V = k.at(3, kBf16, kv), *g2 = k.at(4, kBf16, kv), *kI = k.at(5, kBf16, {B, L, k.c->dI});
        const auto *n_new = (const int32_t*)k.at(6, kI32, {B}), *start = (const int32_t*)k.at(7, kI32, {B});
        return unlocked([&] { return g_fn.append(k.c, (int32_t)L, K, V, g2, kI, n_new, start, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, K, V, kI, ws, stream)
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 7, [](const Args& k) {
        const int some = k.a[2] != Py_None ? 2 : k.a[3] != Py_None ? 3 : 4;
        const int64_t B = k.c->B, L = k.rows(some, "K and V are [B, L, n_kv, d_h], kI [B, L, dI]; at least one of them is wanted");
        const std::initializer_list<int64_t> kv = {B, L, k.c->n_kv, k.c->d_h};
        void *K = k.at(2, kBf16, kv), *V = k.at(3, kBf16, kv), *kI = k.at(4, kBf16, {B, L, k.c->dI});
        return unlocked([&] { return g_fn.read(k.c, (int32_t)L, K, V, kI, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, src_of, share, ws, stream)
PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 6, [](const Args& k) {
        const auto* src = (const int32_t*)k.at(2, kI32, {k.c->B});
        const int32_t share = Args::integer(k.a[3]) != 0;
        return unlocked([&] { return g_fn.fork(k.c, src, share, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, drop, ws, stream)
PyObject* release(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 5, [](const Args& k) {
        const auto* drop = (const int32_t*)k.at(2, kI32, {k.c->B});
        return unlocked([&] { return g_fn.release(k.c, drop, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, live_pages, ws, stream)
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 5, [](const Args& k) {
        auto* live = (int32_t*)k.at(2, kI32, {1});
        return unlocked([&] { return g_fn.compact(k.c, live, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, p, qI, w, bI, scores, row_stride, ws, stream)
PyObject* indexer_scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 10, [](const Args& k) {
        const gsa_params_t* p = k.params(2);
        const int64_t stride = Args::integer(k.a[7]);
        const void* qI = k.at(3, kBf16, {p->B, p->Lq, p->HI, p->dI});
        const auto *w = (const float*)k.at(4, kF32, {p->B, p->Lq, p->HI}), *bI = (const float*)k.at(5, kF32, {p->HI});
        auto* scores = (float*)k.at(6, kF32, {p->B, p->Lq, stride});
        return unlocked([&] { return g_fn.indexer_scores(k.c, p, qI, w, bI, scores, stride, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, p, scores, row_stride, idx, kt, var, ws, stream)
PyObject* topk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 10, [](const Args& k) {
        const gsa_params_t* p = k.params(2);
        const int64_t stride = Args::integer(k.a[4]);
        const auto* scores = (const float*)k.at(3, kF32, {p->B, p->Lq, stride});
        auto *idx = (int32_t*)k.at(5, kI32, {p->B, p->Lq, p->k_max}), *kt = (int32_t*)k.at(6, kI32, {p->B, p->Lq});
        auto* var = (float*)k.at(7, kF32, {p->B, p->Lq});
        return unlocked([&] { return g_fn.topk(k.c, p, scores, stride, idx, kt, var, k.ws, k.ws_bytes, k.stream); });
    });
}
// (c, device, p, Q, g1, idx, kt, out, ws, stream)
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 10, [](const Args& k) {
        const gsa_params_t* p = k.params(2);
        const std::initializer_list<int64_t> heads = {p->B, p->Lq, p->n_h, p->d_h};
        const void *Q = k.at(3, kBf16, heads), *g1 = k.at(4, kBf16, heads);
        const auto *idx = (const int32_t*)k.at(5, kI32, {p->B, p->Lq, p->k_max}), *kt = (const int32_t*)k.at(6, kI32, {p->B, p->Lq});
        void* out = k.at(7, kBf16, heads);
        return unlocked([&] { return g_fn.attn_fwd(k.c, p, Q, g1, idx, kt, out, k.ws, k.ws_bytes, k.stream); });
    });
}

// bind(GsaError, addresses of the nine functions in the order of g_fn)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr Py_ssize_t kFns = sizeof(g_fn) / sizeof(void*);
    if (n != kFns + 1 || !PyExceptionClass_Check(a[0])) {
        PyErr_SetString(PyExc_TypeError, "bind(exception, address, ...)");
        return nullptr;
    }
    void* at[kFns];
    for (Py_ssize_t i = 0; i < kFns; ++i) {
        at[i] = PyLong_AsVoidPtr(a[i + 1]);
        if (!at[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no function");
            return nullptr;
        }
    }
    static_assert(sizeof(g_fn) == sizeof(at), "one pointer each");
    memcpy((void*)&g_fn, at, sizeof(at));
    Py_INCREF(a[0]);
    Py_XSETREF(g_error, a[0]);
    Py_RETURN_NONE;
}

#define GSA_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {GSA_METHOD(call),    GSA_METHOD(bind),           GSA_METHOD(reserve), GSA_METHOD(append), GSA_METHOD(read),     GSA_METHOD(fork),
                         GSA_METHOD(release), GSA_METHOD(compact),        GSA_METHOD(indexer_scores), GSA_METHOD(topk), GSA_METHOD(attn_fwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gsa_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (GSA_BUILT_FOR: the PyTorch and interpreter whose headers this was compiled with, which the binding compares with those that run)
PyMODINIT_FUNC PyInit__gsa_call(void) {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", GSA_BUILT_FOR) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
