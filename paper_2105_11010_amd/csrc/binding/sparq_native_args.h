// What the entry points' marshalling shares: arguments by position and by name, tensors as device buffers, one call of the library.
#pragma once
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "../../../include/sparq.h"

namespace sparq_native {

inline PyObject *mode_type, *desc_type, *error_type;        // SparqMode, SparqConvDesc, SparqError of binding.py

struct PythonError {};                               // a Python exception is set

[[noreturn]] inline void raise(PyObject* type, const char* text) {
    PyErr_SetString(type, text);
    throw PythonError{};
}

// ---- arguments by position and by name ----
template <int N>
struct Signature {
    const char* function;
    const char* names[N];
    int required;
    PyObject* interned[N];
};
template <int N>
void parse(Signature<N>& sig, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames, PyObject* (&out)[N]) {
    if (!sig.interned[0])
        for (int i = 0; i < N; ++i)
            if (!(sig.interned[i] = PyUnicode_InternFromString(sig.names[i]))) throw PythonError{};
    if (nargs > N) {
        PyErr_Format(PyExc_TypeError, "%s() takes at most %d positional arguments but %zd were given", sig.function, N, nargs);
        throw PythonError{};
    }
    for (int i = 0; i < N; ++i) out[i] = i < nargs ? args[i] : nullptr;
    const Py_ssize_t nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < nkw; ++k) {
        PyObject* name = PyTuple_GET_ITEM(kwnames, k);
        int at = -1;
        for (int i = 0; i < N && at < 0; ++i)
            if (name == sig.interned[i]) at = i;
        for (int i = 0; i < N && at < 0; ++i)
            if (PyUnicode_Compare(name, sig.interned[i]) == 0) at = i;
        if (at < 0) {
            PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", sig.function, name);
            throw PythonError{};
        }
        if (out[at]) {
            PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%s'", sig.function, sig.names[at]);
            throw PythonError{};
        }
        out[at] = args[nargs + k];
    }
    for (int i = 0; i < sig.required; ++i)
        if (!out[i]) {
            PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%s'", sig.function, sig.names[i]);
            throw PythonError{};
        }
}
inline bool given(PyObject* o) { return o && o != Py_None; }

// ---- tensors ----
inline const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor, not %s", name, Py_TYPE(o)->tp_name);
        throw PythonError{};
    }
    return THPVariable_Unpack(o);
}
template <class T>
constexpr at::ScalarType kDtype = std::is_same_v<T, uint8_t> ? at::kByte : std::is_same_v<T, int32_t> ? at::kInt : at::kFloat;
template <class T>
T* device_pointer(const at::Tensor& t, const char* name) {
    if (!t.is_cuda() || t.scalar_type() != kDtype<T> || !t.is_contiguous()) {
        PyErr_Format(PyExc_TypeError, "%s must be a contiguous device tensor of dtype %s", name,
                     kDtype<T> == at::kByte ? "torch.uint8" : kDtype<T> == at::kInt ? "torch.int32" : "torch.float32");
        throw PythonError{};
    }
    return static_cast<T*>(t.data_ptr());
}
template <class T>
T* device_pointer(PyObject* o, const char* name) { return given(o) ? device_pointer<T>(tensor(o, name), name) : nullptr; }

// The current device's current stream, as the caller sees it.
inline void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// ---- one call of the library, other Python threads running ----
template <class F>
PyObject* call(const char* what, F&& f) {
    PyThreadState* state = PyEval_SaveThread();
    const sparq_status status = f();
    PyEval_RestoreThread(state);
    if (status == SPARQ_OK) Py_RETURN_NONE;
    PyObject* e = PyObject_CallFunction(error_type, "is", (int)status, what);
    if (e) {
        PyErr_SetObject(error_type, e);
        Py_DECREF(e);
    }
    throw PythonError{};
}
template <PyObject* (*F)(PyObject* const*, Py_ssize_t, PyObject*)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    try {
        return F(args, nargs, kwnames);
    } catch (const PythonError&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

}  // namespace sparq_native
