// What the microscaled entry points' marshalling shares: rows of a matrix, codes with their scales, workspaces.
#pragma once
#include <c10/hip/HIPFunctions.h>

#include "../../../include/sparq_mx.h"
#include "sparq_native_args.h"

namespace sparq_native {

inline decltype(&sparq_mx_code_bytes) code_bytes;        // of the library (bind_mx)
inline decltype(&sparq_mx_scale_bytes) scale_bytes;

[[noreturn]] inline void refuse(PyObject* type, const char* format, const char* name) {
    PyErr_Format(type, format, name);
    throw PythonError{};
}
inline const at::Tensor& on_device(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) refuse(PyExc_TypeError, "%s must be a device tensor", name);
    if (t.get_device() != c10::hip::current_device()) refuse(PyExc_ValueError, "%s must be on the current device", name);
    return t;
}

// Rows of the last axis, of one of the three types: a matrix with any distance between its rows, or a contiguous tensor.
struct Rows {
    void* data = nullptr;
    int64_t rows = 0, length = 0, ld = 0;
    int32_t type = 0;
};
inline Rows rows_of(PyObject* o, const char* name) {
    const at::Tensor& t = on_device(o, name);
    Rows r;
    switch (t.scalar_type()) {
        case at::kFloat: r.type = SPARQ_MX_F32; break;
        case at::kHalf: r.type = SPARQ_MX_F16; break;
        case at::kBFloat16: r.type = SPARQ_MX_BF16; break;
        default: refuse(PyExc_TypeError, "%s must be of dtype torch.float32, torch.float16 or torch.bfloat16", name);
    }
    const int64_t dims = t.dim();
    if (dims < 1) refuse(PyExc_ValueError, "%s must have a last axis", name);
    r.length = t.size(dims - 1);
    if (r.length < 1 || r.length > INT32_MAX) refuse(PyExc_ValueError, "%s must have a last axis of at least one value and fewer than 2^31", name);
    r.rows = t.numel() / r.length;
    r.ld = r.length;
    if (dims == 2) {
        if (r.length > 1 && t.stride(1) != 1) refuse(PyExc_ValueError, "%s must hold the values of a row next to each other", name);
        if (r.rows > 1) r.ld = t.stride(0);
    } else if (!t.is_contiguous()) {
        refuse(PyExc_ValueError, "%s must be a matrix or contiguous", name);
    }
    r.data = t.data_ptr();
    return r;
}
inline Rows rows_like(PyObject* o, const char* name, int64_t rows, int64_t length, int32_t type = -1) {
    const Rows r = rows_of(o, name);
    if (r.rows != rows || r.length != length) {
        PyErr_Format(PyExc_ValueError, "%s must hold %lld rows of %lld", name, (long long)rows, (long long)length);
        throw PythonError{};
    }
    if (type >= 0 && r.type != type) refuse(PyExc_TypeError, "%s must have the type of the call's first tensor", name);
    return r;
}

template <class T>
T* buffer(PyObject* o, const char* name, int64_t elements) {
    if (!given(o)) return nullptr;
    const at::Tensor& t = on_device(o, name);
    T* p = device_pointer<T>(t, name);
    if (t.numel() != elements) {
        PyErr_Format(PyExc_ValueError, "%s must hold %lld elements", name, (long long)elements);
        throw PythonError{};
    }
    return p;
}
struct Coded {
    uint8_t *codes = nullptr, *scales = nullptr;
};
inline Coded coded(PyObject* codes, const char* codes_name, PyObject* scales, const char* scales_name, int64_t rows, int64_t K, int bits) {
    if (given(codes) != given(scales)) refuse(PyExc_ValueError, "%s and its scales go together", codes_name);
    return {buffer<uint8_t>(codes, codes_name, rows * (int64_t)code_bytes((int32_t)K, bits)),
            buffer<uint8_t>(scales, scales_name, rows * (int64_t)scale_bytes((int32_t)K))};
}
struct Scratch {
    void* data = nullptr;
    size_t bytes = 0;
};
inline Scratch scratch(PyObject* o) {
    if (!given(o)) return {};
    const at::Tensor& t = on_device(o, "workspace");
    return {device_pointer<uint8_t>(t, "workspace"), (size_t)t.numel()};
}
inline int32_t integer(PyObject* o, const char* name) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError{};
    if (v < 1 || v > INT32_MAX) refuse(PyExc_ValueError, "%s must be a positive 32-bit number", name);
    return (int32_t)v;
}
inline int32_t function_of(PyObject* o) {
    if (PyUnicode_Check(o)) {
        if (PyUnicode_CompareWithASCIIString(o, "silu") == 0) return SPARQ_MX_SILU;
        if (PyUnicode_CompareWithASCIIString(o, "gelu") == 0) return SPARQ_MX_GELU;
    }
    raise(PyExc_ValueError, "function must be \"silu\" or \"gelu\"");
}

}  // namespace sparq_native
