// CPython module `_block_binding`: the recurrent block's calls without ctypes in between, in the manner of
// layer_binding.cpp: positional arguments in the order of the C functions, addresses as integers or None, the status back.

#include "layer_binding_calls.h"

#include "ctc_block.h"

namespace {

decltype(&ctc_recurrence) g_recurrence;
decltype(&ctc_recurrence_backward) g_recurrence_backward;
decltype(&ctc_block_norm) g_block_norm;
decltype(&ctc_block_norm_backward) g_block_norm_backward;
decltype(&ctc_clear_frames) g_clear_frames;
decltype(&ctc_quantize_weights_i4) g_quantize_weights_i4;
decltype(&ctc_dequantize_weights_i4) g_dequantize_weights_i4;
decltype(&ctc_linear_i4) g_linear_i4;

PyObject* recurrence(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_recurrence, a, n); }
PyObject* recurrence_backward(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_recurrence_backward, a, n); }
PyObject* block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_block_norm, a, n); }
PyObject* block_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_block_norm_backward, a, n); }
PyObject* clear_frames(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_clear_frames, a, n); }
PyObject* quantize_weights_i4(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_quantize_weights_i4, a, n); }
PyObject* dequantize_weights_i4(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_dequantize_weights_i4, a, n); }
PyObject* linear_i4(PyObject*, PyObject* const* a, Py_ssize_t n) { return call(g_linear_i4, a, n); }

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 8) {
        PyErr_Format(PyExc_TypeError, "expected 8 arguments, got %zd", n);
        return nullptr;
    }
    if (!address(a[0], &g_recurrence) || !address(a[1], &g_recurrence_backward) || !address(a[2], &g_block_norm) ||
        !address(a[3], &g_block_norm_backward) || !address(a[4], &g_clear_frames) || !address(a[5], &g_quantize_weights_i4) ||
        !address(a[6], &g_dequantize_weights_i4) || !address(a[7], &g_linear_i4))
        return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"bind", method(bind), METH_FASTCALL, "Addresses of the library's functions, in the order of this module's."},
    {"recurrence", method(recurrence), METH_FASTCALL, nullptr},
    {"recurrence_backward", method(recurrence_backward), METH_FASTCALL, nullptr},
    {"block_norm", method(block_norm), METH_FASTCALL, nullptr},
    {"block_norm_backward", method(block_norm_backward), METH_FASTCALL, nullptr},
    {"clear_frames", method(clear_frames), METH_FASTCALL, nullptr},
    {"quantize_weights_i4", method(quantize_weights_i4), METH_FASTCALL, nullptr},
    {"dequantize_weights_i4", method(dequantize_weights_i4), METH_FASTCALL, nullptr},
    {"linear_i4", method(linear_i4), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_block_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block_binding(void) { return PyModule_Create(&g_module); }
