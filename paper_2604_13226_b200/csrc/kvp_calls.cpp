// The calls on tensors of a decode step on a paged cache, marshalled in C++: a layer's append takes seven tensors and more, and
// looking each up from Python - address, sizes, strides, type, device - costs 0.6 us apiece: an append of one token took 7.5 us
// of host time that way and takes 3.1 this way, 2.5 of them in the library and the driver.
// Nothing is computed here: a call whose tensors fit is handed to the library (whose own checks follow), one whose tensors do
// not fit is given back (-1) to binding.py, which says what is wrong with it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <type_traits>

#include <ATen/core/TensorBase.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kvp.h"

namespace {

decltype(&kvp_cache_append) g_append = nullptr;
decltype(&kvp_cache_attend) g_attend = nullptr;
decltype(&kvp_cache_compact) g_compact = nullptr;
decltype(&kvp_norm_rope) g_norm_rope = nullptr;

struct wanted {
    c10::ScalarType type;
    int device;                    // -1: CPU
    int64_t d;
};

bool on_device(const at::Tensor &t, int device)
{
    return device < 0 ? t.is_cpu() : t.is_cuda() && t.get_device() == device;
}

// [n][heads][d]; n < 0, heads < 0: any, and told.  Written to where p is not const (a lazily cloned tensor then gets memory of its own:
// outputs are asked for in front of inputs, so that one that is both has one address).
template <typename P>
bool rows(PyObject *o, const wanted &w, int64_t &n, int64_t &heads, P *&p, int64_t *stride)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 3 || t.scalar_type() != w.type || t.layout() != c10::kStrided || !on_device(t, w.device)) return false;
    const auto size = t.sizes(), step = t.strides();
    if ((n >= 0 && size[0] != n) || (heads >= 0 && size[1] != heads) || size[2] != w.d || step[2] != 1) return false;
    n = size[0];
    heads = size[1];
    if constexpr (std::is_const_v<P>) p = t.const_data_ptr();
    else p = t.mutable_data_ptr();
    stride[0] = step[0];
    stride[1] = step[1];
    return true;
}

// [n] of int32, or [n][m] with m told
bool ints(PyObject *o, int device, int64_t n, const int32_t *&p, int64_t *cols = nullptr, int64_t *stride = nullptr)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != (cols ? 2 : 1) || t.scalar_type() != c10::kInt || t.layout() != c10::kStrided || !on_device(t, device) || t.size(0) != n) return false;
    if (cols) {
        if (t.size(1) > 1 && t.stride(1) != 1) return false;
        *cols = t.size(1);
        *stride = t.stride(0);
    } else if (n > 1 && t.stride(0) != 1) {
        return false;
    }
    p = static_cast<const int32_t *>(t.const_data_ptr());
    return true;
}

bool vector_of(PyObject *o, const wanted &w, const void *&p)
{
    if (!THPVariable_Check(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 1 || t.scalar_type() != w.type || t.layout() != c10::kStrided || !on_device(t, w.device) || t.size(0) != w.d || t.stride(0) != 1) return false;
    p = t.const_data_ptr();
    return true;
}

// False: an exception is set
bool cache_of(PyObject *const *args, void *&handle, int32_t &layer, bool &fits, wanted &w)
{
    handle = PyLong_AsVoidPtr(args[0]);
    const long number = PyLong_AsLong(args[1]);
    fits = number == (int32_t)number;
    layer = (int32_t)number;
    w.type = PyLong_AsLong(args[2]) == KVP_DTYPE_BF16 ? c10::kBFloat16 : c10::kFloat;
    w.device = (int)PyLong_AsLong(args[3]);
    w.d = PyLong_AsLong(args[4]);
    return !PyErr_Occurred();
}

bool given(PyObject *o) { return o != Py_None; }

// (cache, layer, dtype, device, head_dim, k, v, positions, slots, rope, q, q_out, k_out, q_weight, k_weight, eps, stream) -> status
PyObject *append(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    if (n_args != 17 || !g_append) return PyErr_Format(PyExc_TypeError, "append: %zd arguments", n_args);
    void *handle;
    int32_t layer;
    wanted w;
    bool fits;
    if (!cache_of(args, handle, layer, fits, w)) return nullptr;
    kvp_tokens t = {};
    t.struct_bytes = sizeof t;
    const void *rope = given(args[9]) ? PyLong_AsVoidPtr(args[9]) : nullptr;
    t.eps = PyFloat_AsDouble(args[15]);
    void *stream = given(args[16]) ? PyLong_AsVoidPtr(args[16]) : nullptr;
    if (PyErr_Occurred()) return nullptr;
    int64_t n = -1, hq = -1, hkv = -1;
    try {
        fits = fits && (!given(args[11]) || rows(args[11], w, n, hq, t.q_out, t.q_out_stride)) && (!given(args[12]) || rows(args[12], w, n, hkv, t.k_out, t.k_out_stride)) &&
               rows(args[5], w, n, hkv, t.k, t.k_stride) && rows(args[6], w, n, hkv, t.v, t.v_stride) && n <= INT32_MAX && hkv <= INT32_MAX &&
               (!given(args[7]) || ints(args[7], w.device, n, t.positions)) && ints(args[8], w.device, n, t.slots) &&
               (!given(args[10]) || rows(args[10], w, n, hq, t.q, t.q_stride)) && hq <= INT32_MAX &&
               (!given(args[13]) || vector_of(args[13], w, t.q_weight)) && (!given(args[14]) || vector_of(args[14], w, t.k_weight));
    } catch (...) {                                // a tensor without memory, say
        fits = false;
    }
    if (!fits) return PyLong_FromLong(-1);
    t.n_tokens = (int32_t)n;
    t.n_q_heads = given(args[10]) ? (int32_t)hq : 0;
    t.n_kv_heads = (int32_t)hkv;
    return PyLong_FromLong(g_append((kvp_cache *)handle, layer, &t, (const kvp_rope *)rope, stream));
}

// (cache, layer, dtype, device, head_dim, q heads, q, out, table, lens, first, lse, stream) -> status
PyObject *attend(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    if (n_args != 13 || !g_attend) return PyErr_Format(PyExc_TypeError, "attend: %zd arguments", n_args);
    void *handle;
    int32_t layer;
    wanted w;
    bool fits;
    if (!cache_of(args, handle, layer, fits, w)) return nullptr;
    int64_t hq = PyLong_AsLong(args[5]), n = -1, cols = 0, table_stride = 0, q_stride[2], out_stride[2];
    void *stream = given(args[12]) ? PyLong_AsVoidPtr(args[12]) : nullptr;
    if (PyErr_Occurred()) return nullptr;
    const void *q = nullptr;
    void *out = nullptr;
    const int32_t *table = nullptr, *lens = nullptr, *first = nullptr;
    float *lse = nullptr;
    try {
        fits = fits && rows(args[7], w, n, hq, out, out_stride) && rows(args[6], w, n, hq, q, q_stride) && n <= INT32_MAX &&
               ints(args[8], w.device, n, table, &cols, &table_stride) && cols <= INT32_MAX && ints(args[9], w.device, n, lens) &&
               (!given(args[10]) || ints(args[10], w.device, n, first));
        if (fits && given(args[11])) {
            fits = THPVariable_Check(args[11]);
            if (fits) {
                const at::Tensor &t = THPVariable_Unpack(args[11]);
                fits = t.dim() == 2 && t.scalar_type() == c10::kFloat && t.layout() == c10::kStrided && on_device(t, w.device) && t.size(0) == n && t.size(1) == hq && t.is_contiguous();
                if (fits) lse = static_cast<float *>(t.mutable_data_ptr());
            }
        }
    } catch (...) {
        fits = false;
    }
    if (!fits) return PyLong_FromLong(-1);
    return PyLong_FromLong(g_attend((kvp_cache *)handle, layer, (int32_t)n, q, q_stride, table, table_stride, (int32_t)cols, lens, first,
                                    out, out_stride, lse, stream));
}

// (cache, device, layers, kv heads, table, lens, new_table, kept, n_kept, stream) -> status
PyObject *compact(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    if (n_args != 10 || !g_compact) return PyErr_Format(PyExc_TypeError, "compact: %zd arguments", n_args);
    void *handle = PyLong_AsVoidPtr(args[0]), *stream = given(args[9]) ? PyLong_AsVoidPtr(args[9]) : nullptr;
    const int device = (int)PyLong_AsLong(args[1]);
    const int64_t layers = PyLong_AsLong(args[2]), heads = PyLong_AsLong(args[3]);
    if (PyErr_Occurred()) return nullptr;
    int64_t n = 0, cols = 0, stride = 0, new_cols = 0, new_stride = 0, kept_stride[3] = {0, 0, 0}, most = 0;
    const int32_t *table = nullptr, *lens = nullptr, *new_table = nullptr, *kept = nullptr, *n_kept = nullptr;
    bool fits = THPVariable_Check(args[7]) && THPVariable_Check(args[8]);
    try {
        if (fits) {
            const at::Tensor &t = THPVariable_Unpack(args[7]);
            fits = t.dim() == 4 && t.scalar_type() == c10::kInt && t.layout() == c10::kStrided && on_device(t, device) && (t.size(3) <= 1 || t.stride(3) == 1) &&
                   (t.size(1) == 1 || t.size(1) == layers) && (t.size(2) == 1 || t.size(2) == heads);
            if (fits) {
                n = t.size(0);
                most = t.size(3);
                kept_stride[0] = t.stride(0);
                kept_stride[1] = t.size(1) > 1 ? t.stride(1) : 0;
                kept_stride[2] = t.size(2) > 1 ? t.stride(2) : 0;
                kept = static_cast<const int32_t *>(t.const_data_ptr());
            }
        }
        fits = fits && n <= INT32_MAX && most <= INT32_MAX && ints(args[4], device, n, table, &cols, &stride) && cols <= INT32_MAX && ints(args[5], device, n, lens) &&
               ints(args[6], device, n, new_table, &new_cols, &new_stride) && new_cols <= INT32_MAX && ints(args[8], device, n, n_kept);
    } catch (...) {
        fits = false;
    }
    if (!fits) return PyLong_FromLong(-1);
    return PyLong_FromLong(g_compact((kvp_cache *)handle, (int32_t)n, table, stride, (int32_t)cols, lens, new_table, new_stride, (int32_t)new_cols, kept,
                                     kept_stride, (int32_t)most, n_kept, stream));
}

// (device, q, k, positions, rope, q_out, k_out, q_weight, k_weight, eps, stream) -> status
PyObject *norm_rope(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    if (n_args != 11 || !g_norm_rope) return PyErr_Format(PyExc_TypeError, "norm_rope: %zd arguments", n_args);
    wanted w;
    w.device = (int)PyLong_AsLong(args[0]);
    kvp_tokens t = {};
    t.struct_bytes = sizeof t;
    const void *rope = given(args[4]) ? PyLong_AsVoidPtr(args[4]) : nullptr;
    t.eps = PyFloat_AsDouble(args[9]);
    void *stream = given(args[10]) ? PyLong_AsVoidPtr(args[10]) : nullptr;
    if (PyErr_Occurred()) return nullptr;
    int64_t n = -1, hq = -1, hkv = -1;
    bool fits = true;
    try {
        PyObject *first = given(args[1]) ? args[1] : args[2];
        fits = w.device >= 0 && THPVariable_Check(first);
        if (fits) {
            const at::Tensor &f = THPVariable_Unpack(first);
            w.type = f.scalar_type();
            w.d = f.dim() == 3 ? f.size(2) : -1;
            fits = w.type == c10::kFloat || w.type == c10::kBFloat16;
        }
        fits = fits && (!given(args[5]) || rows(args[5], w, n, hq, t.q_out, t.q_out_stride)) && (!given(args[6]) || rows(args[6], w, n, hkv, t.k_out, t.k_out_stride)) &&
               (!given(args[1]) || rows(args[1], w, n, hq, t.q, t.q_stride)) && (!given(args[2]) || rows(args[2], w, n, hkv, t.k, t.k_stride)) &&
               n <= INT32_MAX && hq <= INT32_MAX && hkv <= INT32_MAX && w.d <= INT32_MAX && (!given(args[3]) || ints(args[3], w.device, n, t.positions)) &&
               (!given(args[7]) || vector_of(args[7], w, t.q_weight)) && (!given(args[8]) || vector_of(args[8], w, t.k_weight));
    } catch (...) {
        fits = false;
    }
    if (!fits) return PyLong_FromLong(-1);
    t.n_tokens = (int32_t)n;
    t.n_q_heads = given(args[1]) ? (int32_t)hq : 0;
    t.n_kv_heads = given(args[2]) ? (int32_t)hkv : 0;
    return PyLong_FromLong(g_norm_rope(w.device, w.type == c10::kBFloat16 ? KVP_DTYPE_BF16 : KVP_DTYPE_F32, (int32_t)w.d, &t, (const kvp_rope *)rope, stream));
}

// addresses of the library's kvp_cache_append, kvp_cache_attend, kvp_cache_compact and kvp_norm_rope
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    if (n_args != 4) return PyErr_Format(PyExc_TypeError, "bind: %zd arguments", n_args);
    g_append = (decltype(g_append))PyLong_AsVoidPtr(args[0]);
    g_attend = (decltype(g_attend))PyLong_AsVoidPtr(args[1]);
    g_compact = (decltype(g_compact))PyLong_AsVoidPtr(args[2]);
    g_norm_rope = (decltype(g_norm_rope))PyLong_AsVoidPtr(args[3]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {{"append", (PyCFunction)(void *)append, METH_FASTCALL, "kvp_cache_append of tensors; -1: they do not fit"},
                           {"attend", (PyCFunction)(void *)attend, METH_FASTCALL, "kvp_cache_attend of tensors; -1: they do not fit"},
                           {"compact", (PyCFunction)(void *)compact, METH_FASTCALL, "kvp_cache_compact of tensors; -1: they do not fit"},
                           {"norm_rope", (PyCFunction)(void *)norm_rope, METH_FASTCALL, "kvp_norm_rope of tensors; -1: they do not fit"},
                           {"bind", (PyCFunction)(void *)bind, METH_FASTCALL, "the library's calls"},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_kvp_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvp_calls(void) { return PyModule_Create(&g_module); }
