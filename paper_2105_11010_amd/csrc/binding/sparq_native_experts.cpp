// Argument marshalling of the entry points of a block with experts (include/sparq_mx_experts.h), in the manner of sparq_native_mx.cpp.
#include "../../../include/sparq_mx_experts.h"

#include "sparq_native_mx_args.h"

namespace {
using namespace sparq_native;

struct Library {
    decltype(&sparq_mx_sort) sort;
    decltype(&sparq_mx_gather) gather;
    decltype(&sparq_mx_combine) combine;
    decltype(&sparq_mx_combine_grad) combine_grad;
    decltype(&sparq_mx_experts_gemm) experts_gemm;
    decltype(&sparq_mx_experts_linear) experts_linear;
    decltype(&sparq_mx_experts_dx) experts_dx;
    decltype(&sparq_mx_experts_dw) experts_dw;
    decltype(&sparq_mx_dropout) dropout;
};
Library lib;

struct Numbers {
    int32_t* data = nullptr;
    int64_t count = 0;
};
Numbers numbers(PyObject* o, const char* name) {
    const at::Tensor& t = on_device(o, name);
    return {device_pointer<int32_t>(t, name), t.numel()};
}
// offsets: one number more than there are experts
Numbers offsets_of(PyObject* o, int32_t& experts) {
    const Numbers n = numbers(o, "offsets");
    if (n.count < 2 || n.count > INT32_MAX) raise(PyExc_ValueError, "offsets must hold one number more than there are experts");
    experts = (int32_t)(n.count - 1);
    return n;
}
// place: [tokens][per]
struct Places {
    int32_t* data = nullptr;
    int32_t per = 0;
};
Places places(PyObject* o, int64_t tokens) {
    const at::Tensor& t = on_device(o, "place");
    if (t.dim() != 2 || t.size(0) != tokens || t.size(1) < 1 || t.size(1) > INT32_MAX) raise(PyExc_ValueError, "place must hold a row of at least one number per token");
    return {device_pointer<int32_t>(t, "place"), (int32_t)t.size(1)};
}
int32_t function_or_none(PyObject* o) { return given(o) ? function_of(o) : (int32_t)SPARQ_MX_NONE; }
uint64_t number64(PyObject* o, const char* name) {
    if (!PyLong_Check(o)) refuse(PyExc_TypeError, "%s must be a whole number", name);
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(PyExc_ValueError, "%s must be a number of 64 bits, not below 0", name);
    }
    return v;
}

PyObject* sort(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<5> sig = {"sparq_mx_sort", {"expert", "offsets", "place", "order", "workspace"}, 3, {}};
    PyObject* a[5];
    parse(sig, args, nargs, kwnames, a);
    const Numbers expert = numbers(a[0], "expert");
    int32_t experts = 0;
    const Numbers offsets = offsets_of(a[1], experts);
    if (!given(a[2])) raise(PyExc_TypeError, "place must be a tensor");
    int32_t *place = buffer<int32_t>(a[2], "place", expert.count), *order = buffer<int32_t>(a[3], "order", expert.count);
    const Scratch ws = scratch(a[4]);
    void* s = stream();
    return call("sparq_mx_sort", [&] { return lib.sort(expert.data, expert.count, experts, offsets.data, place, order, ws.data, ws.bytes, s); });
}

PyObject* gather(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<7> sig = {"sparq_mx_gather", {"x", "place", "y", "codes4", "scales4", "codes8", "scales8"}, 2, {}};
    PyObject* a[7];
    parse(sig, args, nargs, kwnames, a);
    const Rows x = rows_of(a[0], "x");
    const Places place = places(a[1], x.rows);
    if (code_bytes((int32_t)x.length, 4) == 0) raise(PyExc_ValueError, "x must have rows of at most 2^28 values");
    int64_t rows = 0;
    Rows y;
    if (given(a[2])) {
        y = rows_of(a[2], "y");
        rows = y.rows;
        if (y.length != x.length) raise(PyExc_ValueError, "x and y must have rows of the same length");
        if (y.type != x.type) raise(PyExc_TypeError, "y must have the type of the call's first tensor");
    } else if (given(a[3])) {
        rows = on_device(a[3], "codes4").numel() / (int64_t)code_bytes((int32_t)x.length, 4);
    } else if (given(a[5])) {
        rows = on_device(a[5], "codes8").numel() / (int64_t)code_bytes((int32_t)x.length, 8);
    } else {
        raise(PyExc_ValueError, "one of y, codes4 and codes8 must be given");
    }
    const Coded c4 = coded(a[3], "codes4", a[4], "scales4", rows, x.length, 4), c8 = coded(a[5], "codes8", a[6], "scales8", rows, x.length, 8);
    void* s = stream();
    return call("sparq_mx_gather", [&] {
        return lib.gather(x.data, x.type, x.ld, x.rows, (int32_t)x.length, place.data, place.per, y.data, y.ld, c4.codes, c4.scales, c8.codes, c8.scales, rows, s);
    });
}

PyObject* combine(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<5> sig = {"sparq_mx_combine", {"x", "place", "y", "weights", "residual"}, 3, {}};
    PyObject* a[5];
    parse(sig, args, nargs, kwnames, a);
    const Rows y = rows_of(a[2], "y"), x = rows_of(a[0], "x");
    if (y.length != x.length) raise(PyExc_ValueError, "x and y must have rows of the same length");
    if (y.type != x.type) raise(PyExc_TypeError, "y must have the type of the call's first tensor");
    const Places place = places(a[1], y.rows);
    const float* weights = buffer<float>(a[3], "weights", y.rows * place.per);
    const Rows residual = given(a[4]) ? rows_like(a[4], "residual", y.rows, y.length, x.type) : Rows{};
    void* s = stream();
    return call("sparq_mx_combine", [&] {
        return lib.combine(x.data, x.ld, x.rows, place.data, weights, place.per, residual.data, residual.ld, y.data, y.ld, y.type, y.rows, (int32_t)y.length, s);
    });
}

PyObject* combine_grad(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<6> sig = {"sparq_mx_combine_grad", {"dy", "place", "weights", "dx", "x", "dweights"}, 2, {}};
    PyObject* a[6];
    parse(sig, args, nargs, kwnames, a);
    const Rows dy = rows_of(a[0], "dy");
    const Places place = places(a[1], dy.rows);
    const float* weights = buffer<float>(a[2], "weights", dy.rows * place.per);
    if (!given(a[3]) && !given(a[5])) raise(PyExc_ValueError, "one of dx and dweights must be given");
    if (given(a[3]) && !given(a[2])) raise(PyExc_ValueError, "dx without weights");
    if (given(a[5]) != given(a[4])) raise(PyExc_ValueError, "x and dweights go together");
    Rows dx, x;
    int64_t rows = 0;
    if (given(a[4])) {
        x = rows_of(a[4], "x");
        rows = x.rows;
        x = rows_like(a[4], "x", rows, dy.length, dy.type);
    }
    if (given(a[3])) {
        if (!given(a[4])) rows = rows_of(a[3], "dx").rows;
        dx = rows_like(a[3], "dx", rows, dy.length, dy.type);
    }
    float* dweights = buffer<float>(a[5], "dweights", dy.rows * place.per);
    void* s = stream();
    return call("sparq_mx_combine_grad", [&] {
        return lib.combine_grad(dy.data, dy.ld, place.data, weights, place.per, dx.data, dx.ld, x.data, x.ld, rows, dweights, dy.type, dy.rows, (int32_t)dy.length, s);
    });
}

// What the two forms of the experts' product have in common, from argument `at` on: offsets, bias, function, residual, kept_codes, kept_scales, workspace
struct Beside {
    Numbers offsets;
    int32_t experts = 1, function;
    const float* bias;
    Rows residual;
    Coded kept;
    Scratch ws;
};
Beside beside(PyObject** a, const Rows& y) {
    Beside b;
    if (given(a[0])) b.offsets = offsets_of(a[0], b.experts);
    b.bias = buffer<float>(a[1], "bias", b.experts * y.length);
    b.function = function_or_none(a[2]);
    if (given(a[3])) b.residual = rows_like(a[3], "residual", y.rows, y.length, y.type);
    b.kept = coded(a[4], "kept_codes", a[5], "kept_scales", y.rows, y.length, 8);
    b.ws = scratch(a[6]);
    return b;
}

PyObject* experts_gemm(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<13> sig = {"sparq_mx_experts_gemm",
                                {"a_codes", "a_scales", "w_codes", "w_scales", "K", "y", "offsets", "bias", "function", "residual", "kept_codes", "kept_scales", "workspace"},
                                6, {}};
    PyObject* a[13];
    parse(sig, args, nargs, kwnames, a);
    const int32_t K = integer(a[4], "K");
    const Rows y = rows_of(a[5], "y");
    const Beside b = beside(a + 6, y);
    const Coded x = coded(a[0], "a_codes", a[1], "a_scales", y.rows, K, 4), w = coded(a[2], "w_codes", a[3], "w_scales", b.experts * y.length, K, 4);
    void* s = stream();
    return call("sparq_mx_experts_gemm", [&] {
        return lib.experts_gemm(x.codes, x.scales, b.offsets.data, b.experts, w.codes, w.scales, b.bias, b.function, b.residual.data, b.residual.ld, y.data, y.type,
                                y.ld, b.kept.codes, b.kept.scales, y.rows, (int32_t)y.length, K, b.ws.data, b.ws.bytes, s);
    });
}

PyObject* experts_linear(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<11> sig = {"sparq_mx_experts_linear",
                                {"x", "w_codes", "w_scales", "y", "offsets", "bias", "function", "residual", "kept_codes", "kept_scales", "workspace"}, 4, {}};
    PyObject* a[11];
    parse(sig, args, nargs, kwnames, a);
    const Rows x = rows_of(a[0], "x"), y = rows_of(a[3], "y");
    if (y.rows != x.rows) raise(PyExc_ValueError, "x and y must have the same number of rows");
    const Beside b = beside(a + 4, y);
    const Coded w = coded(a[1], "w_codes", a[2], "w_scales", b.experts * y.length, x.length, 4);
    void* s = stream();
    return call("sparq_mx_experts_linear", [&] {
        return lib.experts_linear(x.data, x.type, x.ld, b.offsets.data, b.experts, w.codes, w.scales, b.bias, b.function, b.residual.data, b.residual.ld, y.data,
                                  y.type, y.ld, b.kept.codes, b.kept.scales, x.rows, (int32_t)y.length, (int32_t)x.length, b.ws.data, b.ws.bytes, s);
    });
}

PyObject* experts_dx(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<6> sig = {"sparq_mx_experts_dx", {"dy", "offsets", "w_codes", "w_scales", "dx", "workspace"}, 5, {}};
    PyObject* a[6];
    parse(sig, args, nargs, kwnames, a);
    const Rows dy = rows_of(a[0], "dy"), dx = rows_of(a[4], "dx");
    if (dy.rows != dx.rows) raise(PyExc_ValueError, "dy and dx must have the same number of rows");
    int32_t experts = 0;
    const Numbers offsets = offsets_of(a[1], experts);
    const Coded w = coded(a[2], "w_codes", a[3], "w_scales", experts * dy.length, dx.length, 4);
    const Scratch ws = scratch(a[5]);
    void* s = stream();
    return call("sparq_mx_experts_dx", [&] {
        return lib.experts_dx(dy.data, dy.type, dy.ld, offsets.data, experts, w.codes, w.scales, dx.data, dx.type, dx.ld, dy.rows, (int32_t)dy.length,
                              (int32_t)dx.length, ws.data, ws.bytes, s);
    });
}

PyObject* experts_dw(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<7> sig = {"sparq_mx_experts_dw", {"dy", "offsets", "x_codes", "x_scales", "dw", "db", "workspace"}, 5, {}};
    PyObject* a[7];
    parse(sig, args, nargs, kwnames, a);
    const Rows dy = rows_of(a[0], "dy"), dw = rows_of(a[4], "dw");
    int32_t experts = 0;
    const Numbers offsets = offsets_of(a[1], experts);
    if (dw.rows != experts * dy.length) raise(PyExc_ValueError, "dw must have one row per expert and column of dy");
    const Coded x = coded(a[2], "x_codes", a[3], "x_scales", dy.rows, dw.length, 8);
    float* db = buffer<float>(a[5], "db", experts * dy.length);
    const Scratch ws = scratch(a[6]);
    void* s = stream();
    return call("sparq_mx_experts_dw", [&] {
        return lib.experts_dw(dy.data, dy.type, dy.ld, offsets.data, experts, x.codes, x.scales, dw.data, dw.type, dw.ld, db, dy.rows, (int32_t)dy.length,
                              (int32_t)dw.length, ws.data, ws.bytes, s);
    });
}

PyObject* dropout(PyObject* const* args, Py_ssize_t nargs, PyObject* kwnames) {
    static Signature<7> sig = {"sparq_mx_dropout", {"x", "p", "seed", "y", "offset", "residual", "step"}, 4, {}};
    PyObject* a[7];
    parse(sig, args, nargs, kwnames, a);
    const Rows x = rows_of(a[0], "x");
    const double p = PyFloat_AsDouble(a[1]);
    if (p == -1.0 && PyErr_Occurred()) throw PythonError{};
    const uint64_t seed = number64(a[2], "seed"), offset = given(a[4]) ? number64(a[4], "offset") : 0;
    const Rows y = rows_like(a[3], "y", x.rows, x.length, x.type), residual = given(a[5]) ? rows_like(a[5], "residual", x.rows, x.length, x.type) : Rows{};
    const int64_t* step = buffer<int64_t>(a[6], "step", 1);
    void* s = stream();
    return call("sparq_mx_dropout", [&] {
        return lib.dropout(x.data, x.ld, p, seed, offset, reinterpret_cast<const uint64_t*>(step), residual.data, residual.ld, y.data, y.ld, x.type, x.rows,
                           (int32_t)x.length, s);
    });
}

// bind_experts(addresses): addresses of the library's functions, in Library's order
PyObject* bind_experts(PyObject*, PyObject* list) {
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
    Py_RETURN_NONE;
}

#define SPARQ_MX_METHOD(F, DOC) \
    {"sparq_mx_" #F, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<F>)), METH_FASTCALL | METH_KEYWORDS, "sparq_mx_" #F DOC}
PyMethodDef methods[] = {
    SPARQ_MX_METHOD(sort, "(expert, offsets, place, order=None, workspace=None)\n--\n\n"
                          "Slots sorted by expert: each expert's range of rows, each slot's row (-1: refused), each row's slot."),
    SPARQ_MX_METHOD(gather, "(x, place, y=None, codes4=None, scales4=None, codes8=None, scales8=None)\n--\n\n"
                            "Row place[t][j] of the results = row t of x: as it is, in 4 bits, in 8 bits, any of the three from one pass."),
    SPARQ_MX_METHOD(combine, "(x, place, y, weights=None, residual=None)\n--\n\n"
                             "y[t] = residual[t] + sum_j weights[t][j] x[place[t][j]]; without weights: the gradient of sparq_mx_gather."),
    SPARQ_MX_METHOD(combine_grad, "(dy, place, weights=None, dx=None, x=None, dweights=None)\n--\n\n"
                                  "dx[place[t][j]] = weights[t][j] dy[t] and dweights[t][j] = dy[t] . x[place[t][j]], either or both."),
    SPARQ_MX_METHOD(experts_gemm, "(a_codes, a_scales, w_codes, w_scales, K, y, offsets=None, bias=None, function=None, residual=None, kept_codes=None, "
                                  "kept_scales=None, workspace=None)\n--\n\n"
                                  "y = residual + f(A W[e]^T + bias[e]) over 4-bit operands, each row with its expert's weights (offsets=None: one expert), and\n"
                                  "the 8-bit form of what f is applied to where asked for; function None, \"silu\" or \"gelu\"."),
    SPARQ_MX_METHOD(experts_linear, "(x, w_codes, w_scales, y, offsets=None, bias=None, function=None, residual=None, kept_codes=None, kept_scales=None, "
                                    "workspace=None)\n--\n\ny = residual + f(Q4(x) W[e]^T + bias[e]), x quantised on the way."),
    SPARQ_MX_METHOD(experts_dx, "(dy, offsets, w_codes, w_scales, dx, workspace=None)\n--\n\ndx = dy W[e] over the 4-bit weights of each row's expert."),
    SPARQ_MX_METHOD(experts_dw, "(dy, offsets, x_codes, x_scales, dw, db=None, workspace=None)\n--\n\n"
                                "dw[e] = dy^T X and db[e] = the sum of dy's rows, over expert e's rows and their 8-bit form."),
    SPARQ_MX_METHOD(dropout, "(x, p, seed, y, offset=0, residual=None, step=None)\n--\n\n"
                             "y = residual + x m / (1 - p), the mask m made of seed and offset (+ the number in step); on dy: the backward pass."),
    {"bind_experts", bind_experts, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

}  // namespace

namespace sparq_native {
bool add_experts_methods(PyObject* module) { return PyModule_AddFunctions(module, methods) == 0; }
}  // namespace sparq_native
