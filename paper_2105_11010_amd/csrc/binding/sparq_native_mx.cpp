// Argument marshalling of the microscaled entry points (include/sparq_mx.h), in the manner of sparq_native.cpp: sizes come from
// the tensors' shapes, and what a shape or type shows to be wrong is refused before the library is called.
#include "sparq_native_mx_args.h"

namespace {
using namespace sparq_native;

struct Library {
    decltype(&sparq_mx_quantize) quantize;
    decltype(&sparq_mx_dequantize) dequantize;
    decltype(&sparq_mx_gemm) gemm;
    decltype(&sparq_mx_linear) linear;
    decltype(&sparq_mx_linear_dx) linear_dx;
    decltype(&sparq_mx_linear_dw) linear_dw;
    decltype(&sparq_mx_act) act;
    decltype(&sparq_mx_act_grad) act_grad;
    decltype(&sparq_mx_norm) norm;
    decltype(&sparq_mx_norm_grad) norm_grad;
    decltype(&sparq_mx_code_bytes) code_bytes;
    decltype(&sparq_mx_scale_bytes) scale_bytes;
};
Library lib;

PyObject* quantize(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<5> sig = {"sparq_mx_quantize", {"x", "codes4", "scales4", "codes8", "scales8"}, 1, {}};
    PyObject* a[5];
    parse(sig, args, nargs, kwnames, a);
    const Rows x = rows_of(a[0], "x");
    const Coded c4 = coded(a[1], "codes4", a[2], "scales4", x.rows, x.length, 4), c8 = coded(a[3], "codes8", a[4], "scales8", x.rows, x.length, 8);
    void* s = stream();
    return call("sparq_mx_quantize", [&] {
        return lib.quantize(x.data, x.type, x.ld, x.rows, (int32_t)x.length, c4.codes, c4.scales, c8.codes, c8.scales, s);
    });
}

PyObject* dequantize(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<4> sig = {"sparq_mx_dequantize", {"codes", "scales", "bits", "y"}, 4, {}};
    PyObject* a[4];
    parse(sig, args, nargs, kwnames, a);
    const int32_t bits = integer(a[2], "bits");
    if (bits != 4 && bits != 8) raise(PyExc_ValueError, "bits must be 4 or 8");
    const Rows y = rows_of(a[3], "y");
    const Coded c = coded(a[0], "codes", a[1], "scales", y.rows, y.length, bits);
    void* s = stream();
    return call("sparq_mx_dequantize", [&] { return lib.dequantize(c.codes, c.scales, bits, y.data, y.type, y.ld, y.rows, (int32_t)y.length, s); });
}

PyObject* gemm(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<8> sig = {"sparq_mx_gemm", {"a_codes", "a_scales", "w_codes", "w_scales", "K", "y", "bias", "workspace"}, 6, {}};
    PyObject* a[8];
    parse(sig, args, nargs, kwnames, a);
    const int32_t K = integer(a[4], "K");
    const Rows y = rows_of(a[5], "y");
    const Coded x = coded(a[0], "a_codes", a[1], "a_scales", y.rows, K, 4), w = coded(a[2], "w_codes", a[3], "w_scales", y.length, K, 4);
    const float* bias = buffer<float>(a[6], "bias", y.length);
    const Scratch ws = scratch(a[7]);
    void* s = stream();
    return call("sparq_mx_gemm", [&] {
        return lib.gemm(x.codes, x.scales, w.codes, w.scales, bias, y.data, y.type, y.ld, y.rows, (int32_t)y.length, K, ws.data, ws.bytes, s);
    });
}

PyObject* linear(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<6> sig = {"sparq_mx_linear", {"x", "w_codes", "w_scales", "y", "bias", "workspace"}, 4, {}};
    PyObject* a[6];
    parse(sig, args, nargs, kwnames, a);
    const Rows x = rows_of(a[0], "x"), y = rows_of(a[3], "y");
    if (y.rows != x.rows) raise(PyExc_ValueError, "x and y must have the same number of rows");
    const Coded w = coded(a[1], "w_codes", a[2], "w_scales", y.length, x.length, 4);
    const float* bias = buffer<float>(a[4], "bias", y.length);
    const Scratch ws = scratch(a[5]);
    void* s = stream();
    return call("sparq_mx_linear", [&] {
        return lib.linear(x.data, x.type, x.ld, w.codes, w.scales, bias, y.data, y.type, y.ld, x.rows, (int32_t)y.length, (int32_t)x.length, ws.data,
                          ws.bytes, s);
    });
}

PyObject* linear_dx(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<5> sig = {"sparq_mx_linear_dx", {"dy", "w_codes", "w_scales", "dx", "workspace"}, 4, {}};
    PyObject* a[5];
    parse(sig, args, nargs, kwnames, a);
    const Rows dy = rows_of(a[0], "dy"), dx = rows_of(a[3], "dx");
    if (dy.rows != dx.rows) raise(PyExc_ValueError, "dy and dx must have the same number of rows");
    const Coded w = coded(a[1], "w_codes", a[2], "w_scales", dy.length, dx.length, 4);
    const Scratch ws = scratch(a[4]);
    void* s = stream();
    return call("sparq_mx_linear_dx", [&] {
        return lib.linear_dx(dy.data, dy.type, dy.ld, w.codes, w.scales, dx.data, dx.type, dx.ld, dy.rows, (int32_t)dy.length, (int32_t)dx.length,
                             ws.data, ws.bytes, s);
    });
}

PyObject* linear_dw(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<6> sig = {"sparq_mx_linear_dw", {"dy", "x_codes", "x_scales", "dw", "db", "workspace"}, 4, {}};
    PyObject* a[6];
    parse(sig, args, nargs, kwnames, a);
    const Rows dy = rows_of(a[0], "dy"), dw = rows_of(a[3], "dw");
    if (dw.rows != dy.length) raise(PyExc_ValueError, "dw must have one row per column of dy");
    const Coded x = coded(a[1], "x_codes", a[2], "x_scales", dy.rows, dw.length, 8);
    float* db = buffer<float>(a[4], "db", dy.length);
    const Scratch ws = scratch(a[5]);
    void* s = stream();
    return call("sparq_mx_linear_dw", [&] {
        return lib.linear_dw(dy.data, dy.type, dy.ld, x.codes, x.scales, dw.data, dw.type, dw.ld, db, dy.rows, (int32_t)dy.length,
                             (int32_t)dw.length, ws.data, ws.bytes, s);
    });
}

PyObject* act(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<8> sig = {"sparq_mx_act", {"function", "gate", "y", "up", "gate_codes", "gate_scales", "up_codes", "up_scales"}, 3, {}};
    PyObject* a[8];
    parse(sig, args, nargs, kwnames, a);
    const int32_t f = function_of(a[0]);
    const Rows gate = rows_of(a[1], "gate"), y = rows_like(a[2], "y", gate.rows, gate.length, gate.type);
    const Rows up = given(a[3]) ? rows_like(a[3], "up", gate.rows, gate.length, gate.type) : Rows{};
    const Coded g = coded(a[4], "gate_codes", a[5], "gate_scales", gate.rows, gate.length, 8);
    const Coded u = coded(a[6], "up_codes", a[7], "up_scales", gate.rows, gate.length, 8);
    if (given(a[6]) && !given(a[3])) raise(PyExc_ValueError, "up_codes without up");
    void* s = stream();
    return call("sparq_mx_act", [&] {
        return lib.act(f, gate.data, gate.ld, up.data, up.ld, y.data, y.ld, gate.type, g.codes, g.scales, u.codes, u.scales, gate.rows,
                       (int32_t)gate.length, s);
    });
}

PyObject* act_grad(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<8> sig = {"sparq_mx_act_grad", {"function", "dy", "gate_codes", "gate_scales", "dgate", "up_codes", "up_scales", "dup"}, 5, {}};
    PyObject* a[8];
    parse(sig, args, nargs, kwnames, a);
    const int32_t f = function_of(a[0]);
    const Rows dy = rows_of(a[1], "dy"), dgate = rows_like(a[4], "dgate", dy.rows, dy.length, dy.type);
    if (given(a[5]) != given(a[7])) raise(PyExc_ValueError, "up_codes and dup go together");
    const Rows dup = given(a[7]) ? rows_like(a[7], "dup", dy.rows, dy.length, dy.type) : Rows{};
    const Coded g = coded(a[2], "gate_codes", a[3], "gate_scales", dy.rows, dy.length, 8);
    const Coded u = coded(a[5], "up_codes", a[6], "up_scales", dy.rows, dy.length, 8);
    void* s = stream();
    return call("sparq_mx_act_grad", [&] {
        return lib.act_grad(f, dy.data, dy.ld, g.codes, g.scales, u.codes, u.scales, dgate.data, dgate.ld, dup.data, dup.ld, dy.type, dy.rows,
                            (int32_t)dy.length, s);
    });
}

PyObject* norm(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<9> sig = {"sparq_mx_norm", {"x", "gamma", "beta", "eps", "y", "mean", "rstd", "codes", "scales"}, 5, {}};
    PyObject* a[9];
    parse(sig, args, nargs, kwnames, a);
    const Rows x = rows_of(a[0], "x"), y = rows_like(a[4], "y", x.rows, x.length, x.type);
    const float *gamma = buffer<float>(a[1], "gamma", x.length), *beta = buffer<float>(a[2], "beta", x.length);
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError{};
    float *mean = buffer<float>(a[5], "mean", x.rows), *rstd = buffer<float>(a[6], "rstd", x.rows);
    const Coded c = coded(a[7], "codes", a[8], "scales", x.rows, x.length, 8);
    void* s = stream();
    return call("sparq_mx_norm", [&] {
        return lib.norm(x.data, x.ld, gamma, beta, (float)eps, y.data, y.ld, x.type, mean, rstd, c.codes, c.scales, x.rows, (int32_t)x.length, s);
    });
}

PyObject* norm_grad(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<10> sig = {"sparq_mx_norm_grad", {"dy", "codes", "scales", "mean", "rstd", "gamma", "dx", "dgamma", "dbeta", "workspace"}, 7, {}};
    PyObject* a[10];
    parse(sig, args, nargs, kwnames, a);
    const Rows dy = rows_of(a[0], "dy"), dx = rows_like(a[6], "dx", dy.rows, dy.length, dy.type);
    const Coded c = coded(a[1], "codes", a[2], "scales", dy.rows, dy.length, 8);
    const float *mean = buffer<float>(a[3], "mean", dy.rows), *rstd = buffer<float>(a[4], "rstd", dy.rows);
    const float* gamma = buffer<float>(a[5], "gamma", dy.length);
    float *dgamma = buffer<float>(a[7], "dgamma", dy.length), *dbeta = buffer<float>(a[8], "dbeta", dy.length);
    const Scratch ws = scratch(a[9]);
    void* s = stream();
    return call("sparq_mx_norm_grad", [&] {
        return lib.norm_grad(dy.data, dy.ld, c.codes, c.scales, mean, rstd, gamma, dx.data, dx.ld, dy.type, dgamma, dbeta, dy.rows,
                             (int32_t)dy.length, ws.data, ws.bytes, s);
    });
}

// bind_mx(addresses): addresses of the library's functions, in Library's order
PyObject* bind_mx(PyObject*, PyObject* list) {
    constexpr Py_ssize_t n = sizeof(Library) / sizeof(void*);
    if (!PyTuple_Check(list) || PyTuple_GET_SIZE(list) != n) {
        PyErr_SetString(PyExc_ValueError, "one address per function");
        return nullptr;
    }
    void* addresses[n];
    for (Py_ssize_t i = 0; i < n; ++i) {
        addresses[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(list, i));
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&lib, addresses, sizeof(lib));
    code_bytes = lib.code_bytes;
    scale_bytes = lib.scale_bytes;
    Py_RETURN_NONE;
}

#define SPARQ_MX_METHOD(F, DOC) \
    {"sparq_mx_" #F, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<F>)), METH_FASTCALL | METH_KEYWORDS, "sparq_mx_" #F DOC}
PyMethodDef methods[] = {
    SPARQ_MX_METHOD(quantize, "(x, codes4=None, scales4=None, codes8=None, scales8=None)\n--\n\n"
                              "Codes and scales of x's rows (its last axis): the 4-bit form, the 8-bit form, or both from one pass."),
    SPARQ_MX_METHOD(dequantize, "(codes, scales, bits, y)\n--\n\ny = the values that codes and scales stand for."),
    SPARQ_MX_METHOD(gemm, "(a_codes, a_scales, w_codes, w_scales, K, y, bias=None, workspace=None)\n--\n\n"
                          "y = A W^T + bias over 4-bit operands with rows of K values."),
    SPARQ_MX_METHOD(linear, "(x, w_codes, w_scales, y, bias=None, workspace=None)\n--\n\ny = Q4(x) W^T + bias, x quantised on the way."),
    SPARQ_MX_METHOD(linear_dx, "(dy, w_codes, w_scales, dx, workspace=None)\n--\n\ndx = dy W over the 4-bit weights."),
    SPARQ_MX_METHOD(linear_dw, "(dy, x_codes, x_scales, dw, db=None, workspace=None)\n--\n\n"
                               "dw = dy^T X over the 8-bit checkpoint of the layer's input, db = the sum of dy's rows."),
    SPARQ_MX_METHOD(act, "(function, gate, y, up=None, gate_codes=None, gate_scales=None, up_codes=None, up_scales=None)\n--\n\n"
                         "y = f(gate) * up (up=None: f(gate)), with the inputs' 8-bit checkpoints where asked for; function \"silu\" or \"gelu\"."),
    SPARQ_MX_METHOD(act_grad, "(function, dy, gate_codes, gate_scales, dgate, up_codes=None, up_scales=None, dup=None)\n--\n\n"
                              "dgate and dup from the checkpoints sparq_mx_act wrote."),
    SPARQ_MX_METHOD(norm, "(x, gamma, beta, eps, y, mean=None, rstd=None, codes=None, scales=None)\n--\n\n"
                          "Layer norm over the last axis, with its rows' statistics and x's 8-bit checkpoint where asked for."),
    SPARQ_MX_METHOD(norm_grad, "(dy, codes, scales, mean, rstd, gamma, dx, dgamma=None, dbeta=None, workspace=None)\n--\n\n"
                               "dx and the weights' gradients from what sparq_mx_norm kept."),
    {"bind_mx", bind_mx, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

}  // namespace

namespace sparq_native {
bool add_mx_methods(PyObject* module) { return PyModule_AddFunctions(module, methods) == 0; }
}  // namespace sparq_native
