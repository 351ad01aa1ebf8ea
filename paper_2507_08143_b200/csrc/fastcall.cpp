// Argument checks and marshalling of the paged-cache entry points for Python, compiled.
//
// Decoding calls the attention once per layer and token, and one such call is about 10 us of work on the GPU; reading shapes,
// strides and pointers of ten tensors from Python and passing them through ctypes took 22 us of host time, this takes 2.  The functions
// make the same calls of the C ABI that ctypes would (their addresses come from the loaded library, see bind()).
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "compactor.h"

namespace {

decltype(&compactor_paged_fill) g_fill = nullptr;
decltype(&compactor_paged_attention) g_attention = nullptr;
decltype(&compactor_paged_evict) g_evict = nullptr;

struct Refused {};                       // a Python error has been set

[[noreturn]] void refuse(PyObject* type, const char* name, const char* what) {
    PyErr_Format(type, "%s: %s", name, what);
    throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, name, "a tensor is expected");
    return THPVariable_Unpack(o);
}

// The cache's device, seen from a call: every tensor has to live there, and it has to be the current one.
struct Call {
    const compactor_paged_cache* cache;
    int device;                          // -1: not a CUDA device
    const char* stray = nullptr;         // the first tensor that lives on another device

    void at_home(const at::Tensor& t, const char* name) {
        const int d = t.is_cuda() ? t.get_device() : -1;
        if (d != device && stray == nullptr) stray = name;
    }
    // bf16 [batch, heads, d], contiguous along d
    compactor_rows rows(PyObject* o, int64_t heads, const char* name) {
        if (o == Py_None) return {nullptr, 0, 0};
        const at::Tensor& t = tensor(o, name);
        if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || t.size(0) != cache->batch || t.size(1) != heads ||
            t.size(2) != cache->d || t.stride(2) != 1)
            refuse(PyExc_ValueError, name, "bf16 [batch, heads, d] of this cache, contiguous along the last axis, is expected");
        at_home(t, name);
        return {t.data_ptr(), t.stride(0), t.stride(1)};
    }
    template <typename T>
    T* flat(PyObject* o, at::ScalarType type, int64_t n, const char* name, const char* what) {
        if (o == Py_None) return nullptr;
        const at::Tensor& t = tensor(o, name);
        if (t.scalar_type() != type || t.numel() != n || !t.is_contiguous()) refuse(PyExc_ValueError, name, what);
        at_home(t, name);
        return static_cast<T*>(t.data_ptr());
    }
    int32_t* per_unit(PyObject* o, const char* name) {
        return flat<int32_t>(o, at::kInt, (int64_t)cache->layers * cache->heads * cache->batch, name,
                             "contiguous int32, one entry per (layer, head, sequence), is expected");
    }
    int32_t* per_sequence(PyObject* o, const char* name) {
        return flat<int32_t>(o, at::kInt, cache->batch, name, "contiguous int32 [batch] is expected");
    }
    // bf16 [layers, heads, tokens, d], contiguous along d
    compactor_mat mat(PyObject* o, const compactor_shape* s, const char* name) {
        const at::Tensor& t = tensor(o, name);
        if (t.scalar_type() != at::kBFloat16 || t.dim() != 4 || t.size(0) != s->layers || t.size(1) != s->heads ||
            t.size(2) != s->cu_seqlens[s->batch] || t.size(3) != s->d || t.stride(3) != 1)
            refuse(PyExc_ValueError, name, "bf16 [layers, heads, total tokens, d] of this shape, contiguous along the last axis, is expected");
        at_home(t, name);
        return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
    }
    // Last of all checks: the stream to launch on.
    void* stream() {
        if (device < 0 || c10::cuda::current_device() != device) {
            PyErr_SetString(PyExc_ValueError, "the cache does not live on the current CUDA device");
            throw Refused();
        }
        if (stray != nullptr) refuse(PyExc_ValueError, stray, "lives on another device than the cache");
        return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    }
};

long long integer(PyObject* o) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Refused();
    return x;
}
int32_t integer32(PyObject* o, const char* name) {
    const long long x = integer(o);
    if (x < INT32_MIN || x > INT32_MAX) refuse(PyExc_OverflowError, name, "does not fit 32 bits");
    return (int32_t)x;
}
template <typename T> const T* address(PyObject* o) { return reinterpret_cast<const T*>((uintptr_t)integer(o)); }

// Runs f and turns what it throws into a Python error.
template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F f) {
    if (got != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong(f());
    } catch (const Refused&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// attention(cache, device, layer, options, q, lengths, out, workspace, k_new, v_new, new_positions, lse_out, status)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        Call c{address<compactor_paged_cache>(a[0]), (int)integer(a[1])};
        const int32_t layer = integer32(a[2], "layer");
        const auto* opt = address<compactor_decode_options>(a[3]);
        const int64_t q_heads = (int64_t)c.cache->heads * opt->q_per_kv;
        if (a[4] == Py_None || a[5] == Py_None || a[6] == Py_None) refuse(PyExc_TypeError, "q, lengths, out", "tensors are expected");
        const compactor_rows q = c.rows(a[4], q_heads, "q");
        const int32_t* lengths = c.per_unit(a[5], "lengths");
        const compactor_rows out = c.rows(a[6], q_heads, "out");
        const at::Tensor& ws = tensor(a[7], "workspace");
        if (!ws.is_contiguous()) refuse(PyExc_ValueError, "workspace", "a contiguous tensor is expected");
        c.at_home(ws, "workspace");
        if ((a[8] == Py_None) != (a[9] == Py_None)) refuse(PyExc_ValueError, "k_new, v_new", "come together");
        const compactor_rows kn = c.rows(a[8], c.cache->heads, "k_new"), vn = c.rows(a[9], c.cache->heads, "v_new");
        const int32_t* pos = c.per_sequence(a[10], "new_positions");
        float* lse = c.flat<float>(a[11], at::kFloat, c.cache->batch * q_heads, "lse_out", "contiguous fp32 [batch, heads * q_per_kv] is expected");
        int32_t* status = c.per_unit(a[12], "status");
        return g_attention(c.cache, layer, opt, q, kn, vn, pos, lengths, out, lse, status, ws.data_ptr(), ws.nbytes(), c.stream());
    });
}

// fill(cache, device, first_layer, shape, k_cache, v_cache, keep_counts, idx, head_offsets, mass_in, first_position, lengths, lengths_out, status)
PyObject* fill(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 14, [&] {
        Call c{address<compactor_paged_cache>(a[0]), (int)integer(a[1])};
        const int32_t first_layer = integer32(a[2], "first_layer");
        const auto* shape = address<compactor_shape>(a[3]);
        const compactor_mat k = c.mat(a[4], shape, "k_cache"), v = c.mat(a[5], shape, "v_cache");
        PyObject* seq = PySequence_Fast(a[6], "keep_counts: a sequence of integers is expected");
        if (seq == nullptr) throw Refused();
        struct Held { PyObject* o; ~Held() { Py_DECREF(o); } } held{seq};
        if (PySequence_Fast_GET_SIZE(seq) != shape->batch) refuse(PyExc_ValueError, "keep_counts", "one per sequence is expected");
        std::vector<int32_t> keep(shape->batch);
        int64_t kept = 0;
        for (int b = 0; b < shape->batch; ++b) {
            keep[b] = integer32(PySequence_Fast_GET_ITEM(seq, b), "keep_counts");
            kept += keep[b];
        }
        const int64_t lh = (int64_t)shape->layers * shape->heads;
        const int32_t* idx = c.flat<int32_t>(a[7], at::kInt, lh * kept, "idx", "contiguous int32, one entry per kept row, is expected");
        const int32_t* offs = c.flat<int32_t>(a[8], at::kInt, (int64_t)shape->layers * shape->batch * (shape->heads + 1), "head_offsets",
                                              "contiguous int32 [layers, batch, heads + 1] is expected");
        const float* mass = c.flat<float>(a[9], at::kFloat, lh * shape->cu_seqlens[shape->batch], "mass_in",
                                          "contiguous fp32 [layers, heads, total tokens] is expected");
        const int32_t* pos = c.per_sequence(a[10], "first_position");
        const int32_t* lengths = c.per_unit(a[11], "lengths");
        int32_t* lengths_out = c.per_unit(a[12], "lengths_out");
        int32_t* status = c.per_unit(a[13], "status");
        return g_fill(c.cache, first_layer, shape, k, v, idx, offs, keep.data(), mass, pos, lengths, lengths_out, status, c.stream());
    });
}

// evict(cache, device, first_layer, layers, lengths, budgets, next_position, recent, max_length, lengths_out, status)
PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        Call c{address<compactor_paged_cache>(a[0]), (int)integer(a[1])};
        const int32_t first_layer = integer32(a[2], "first_layer"), layers = integer32(a[3], "layers");
        if (a[4] == Py_None || a[5] == Py_None || a[9] == Py_None) refuse(PyExc_TypeError, "lengths, budgets, lengths_out", "tensors are expected");
        const int32_t* lengths = c.per_unit(a[4], "lengths");
        const int32_t* budgets = c.per_unit(a[5], "budgets");
        const int32_t* next = c.per_sequence(a[6], "next_position");
        const int32_t recent = integer32(a[7], "recent"), max_length = integer32(a[8], "max_length");
        int32_t* lengths_out = c.per_unit(a[9], "lengths_out");
        int32_t* status = c.per_unit(a[10], "status");
        return g_evict(c.cache, first_layer, layers, lengths, budgets, next, recent, max_length, lengths_out, status, c.stream());
    });
}

// bind(fill, attention, evict): addresses of the library's entry points
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 3, [&] {
        g_fill = reinterpret_cast<decltype(g_fill)>((uintptr_t)integer(a[0]));
        g_attention = reinterpret_cast<decltype(g_attention)>((uintptr_t)integer(a[1]));
        g_evict = reinterpret_cast<decltype(g_evict)>((uintptr_t)integer(a[2]));
        return 0;
    });
}

PyMethodDef g_methods[] = {
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attention)), METH_FASTCALL, nullptr},
    {"fill", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(fill)), METH_FASTCALL, nullptr},
    {"evict", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(evict)), METH_FASTCALL, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&g_module); }
