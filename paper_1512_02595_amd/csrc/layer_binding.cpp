// CPython module `_layer_binding`: the output layer's calls without ctypes in between (as binding.cpp does it for the
// CTC path's; a call through ctypes takes ten microseconds, longer than most of these take on the GPU).
//
// The functions take positional arguments only, in the order of the C functions, addresses as integers or None, and
// return the status.  `bind` is given the addresses of the library's functions.

#include "layer_binding_calls.h"

namespace {

decltype(&ctc_pack_frames) g_pack_frames;
decltype(&ctc_quantize_rows) g_quantize_rows;
decltype(&ctc_dequantize_rows) g_dequantize_rows;
decltype(&ctc_rms_norm_i8) g_rms_norm_i8;
decltype(&ctc_rms_norm_backward) g_rms_norm_backward;
decltype(&ctc_linear_i8) g_linear_i8;
decltype(&ctc_weight_gradient_i8) g_weight_gradient_i8;

PyObject* pack_frames(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_pack_frames, a, n); }
PyObject* quantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_quantize_rows, a, n); }
PyObject* dequantize_rows(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_dequantize_rows, a, n); }
PyObject* rms_norm_i8(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_rms_norm_i8, a, n); }
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_rms_norm_backward, a, n); }
PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_linear_i8, a, n); }
PyObject* weight_gradient_i8(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_weight_gradient_i8, a, n); }

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
