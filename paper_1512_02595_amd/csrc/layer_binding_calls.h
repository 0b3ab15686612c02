// What the modules that call the library share: arguments from Python to a C function's types, and its status back.
#ifndef LAYER_BINDING_CALLS_H
#define LAYER_BINDING_CALLS_H

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstdint>
#include <tuple>
#include <utility>

#include "ctc_layer.h"

namespace {

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

template <typename F> bool address(PyObject* o, F* out)
{
    void* p = PyLong_AsVoidPtr(o);
    *out = reinterpret_cast<F>(p);
    return p != nullptr || !PyErr_Occurred();
}

using Fast = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyCFunction method(Fast f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

}  // namespace

#endif  // LAYER_BINDING_CALLS_H
