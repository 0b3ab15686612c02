// CPython module `_layer_binding`: the output layer's calls without ctypes in between (as binding.cpp does it for the
// CTC path's; a call through ctypes takes ten microseconds, longer than most of these take on the GPU).
//
// The functions take positional arguments only, in the order of the C functions, addresses as integers or None, and
// return the status.  `bind` is given the addresses of the library's functions.

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <tuple>
#include <utility>

#include "ctc_layer.h"

namespace {

decltype(&ctc_pack_frames) g_pack_frames;
decltype(&ctc_quantize_rows) g_quantize_rows;
decltype(&ctc_dequantize_rows) g_dequantize_rows;
decltype(&ctc_rms_norm_i8) g_rms_norm_i8;
decltype(&ctc_rms_norm_backward) g_rms_norm_backward;
decltype(&ctc_linear_i8) g_linear_i8;
decltype(&ctc_weight_gradient_i8) g_weight_gradient_i8;

// One argument of a call, taken as the C type that the function has there.
bool take(PyObject* o, int* out)
{
    PyObject* index = PyNumber_Index(o);
    if (!index) return false;
    const long v = PyLong_AsLong(index);
    Py_DECREF(index);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v < INT32_MIN || v > INT32_MAX) {
        PyErr_SetString(PyExc_OverflowError, "a size is out of a 32-bit integer's range");
        return false;
    }
    *out = static_cast<int>(v);
    return true;
}
bool take(PyObject* o, ctc_dtype_t* out)
{
    int v;
    if (!take(o, &v)) return false;
    *out = static_cast<ctc_dtype_t>(v);
    return true;
}
bool take(PyObject* o, float* out)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) return false;
    *out = static_cast<float>(v);
    return true;
}
bool take(PyObject* o, size_t* out)
{
    *out = PyLong_AsSize_t(o);
    return *out != static_cast<size_t>(-1) || !PyErr_Occurred();
}
template <typename T> bool take(PyObject* o, T** out)                       // (None is the null pointer)
{
    void* p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
    *out = static_cast<T*>(p);
    return p || !PyErr_Occurred();
}

template <typename... Args, size_t... I>
PyObject* call_with(ctc_status_t (*f)(Args...), PyObject* const* a, Py_ssize_t n, std::index_sequence<I...>)
{
    if (n != static_cast<Py_ssize_t>(sizeof...(Args))) {
        PyErr_Format(PyExc_TypeError, "expected %zu arguments, got %zd", sizeof...(Args), n);
        return nullptr;
    }
    std::tuple<Args...> args;
    if (!(take(a[I], &std::get<I>(args)) && ...)) return nullptr;
    ctc_status_t st;
    Py_BEGIN_ALLOW_THREADS
    st = f(std::get<I>(args)...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}
template <typename... Args> PyObject* call(ctc_status_t (*f)(Args...), PyObject* const* a, Py_ssize_t n)
{
    return call_with(f, a, n, std::index_sequence_for<Args...>());
}

PyObject* pack_frames(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_pack_frames, a, n); }
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_quantize_rows, a, n); }
PyObject* dequantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_dequantize_rows, a, n); }
PyObject* rms_norm_i8(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_rms_norm_i8, a, n); }
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_rms_norm_backward, a, n); }
PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_linear_i8, a, n); }
PyObject* weight_gradient_i8(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_weight_gradient_i8, a, n); }

template <typename F> bool address(PyObject* o, F* out)
{
    void* p = PyLong_AsVoidPtr(o);
    *out = reinterpret_cast<F>(p);
    return p != nullptr || !PyErr_Occurred();
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 7) {
        PyErr_Format(PyExc_TypeError, "expected 7 arguments, got %zd", n);
        return nullptr;
    }
    if (!address(a[0], &g_pack_frames) || !address(a[1], &g_quantize_rows) || !address(a[2], &g_dequantize_rows) ||
        !address(a[3], &g_rms_norm_i8) || !address(a[4], &g_rms_norm_backward) || !address(a[5], &g_linear_i8) ||
        !address(a[6], &g_weight_gradient_i8))
        return nullptr;
    Py_RETURN_NONE;
}

using Fast = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyCFunction method(Fast f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef g_methods[] = {
    {"bind", method(bind), METH_FASTCALL, "Addresses of the library's functions, in the order of this module's."},
    {"pack_frames", method(pack_frames), METH_FASTCALL, nullptr},
    {"quantize_rows", method(quantize_rows), METH_FASTCALL, nullptr},
    {"dequantize_rows", method(dequantize_rows), METH_FASTCALL, nullptr},
    {"rms_norm_i8", method(rms_norm_i8), METH_FASTCALL, nullptr},
    {"rms_norm_backward", method(rms_norm_backward), METH_FASTCALL, nullptr},
    {"linear_i8", method(linear_i8), METH_FASTCALL, nullptr},
    {"weight_gradient_i8", method(weight_gradient_i8), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_layer_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_binding(void) { return PyModule_Create(&g_module); }
