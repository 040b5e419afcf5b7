// Shared by the two halves of the Python module _launch: calls of the ternary product (launch.cpp) and of the operators around it
// (launch_ops.cpp).
#pragma once
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

namespace launch {

// An attribute that is an int; false (no error set) if it is not there or something else.
inline bool int_attr(PyObject *o, PyObject *name, unsigned long long *out)
{
    PyObject *v = PyObject_GetAttr(o, name);
    const bool ok = v != nullptr && PyLong_CheckExact(v);
    if (ok) *out = PyLong_AsUnsignedLongLong(v);
    Py_XDECREF(v);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return ok;
}

inline bool modes_set()
{
    return at::impl::PythonTorchFunctionTLS::stack_len() > 0 || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

struct WithoutGil {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

extern PyMethodDef ops_methods[];   // launch_ops.cpp; ends with an empty one
bool ops_init();                    // names it looks attributes up by

}  // namespace launch
