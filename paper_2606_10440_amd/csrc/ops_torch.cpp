// The operators' binding to torch tensors: checks them against what the C ABI
// takes, makes results and workspaces with torch's allocator, and enqueues on
// the current stream of the tensors' GPU.
//
// It is in C++ because the host's part of a small call is all of its time:
// quantising 16 x 4096 takes the GPU 2.7 us and the host 4.8 us, most of them
// the launch; the same in Python by way of ctypes took 7.2 us (3.3 for the C
// call, 1.2 for each new tensor).  A router's call: 7.0 us, 10.4 in Python.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <string>

#include "simgpu_ops.h"

namespace {

using at::Tensor;

PyObject *g_error, *g_mx4, *g_routes;  // SimError, Mx4, Routes

// The library's functions, as it was loaded for the rest of the package.
#define SIM_OPS_CALLS(X)                                                                                            \
    X(sim_mx4_quantize) X(sim_mx4_dequantize) X(sim_mx4_matmul) X(sim_mx4_linear_workspace) X(sim_mx4_linear)       \
        X(sim_mx4_linear_grad_workspace) X(sim_mx4_linear_grad) X(sim_moe_route_workspace) X(sim_moe_route)         \
            X(sim_moe_route_grad) X(sim_moe_layer_workspace) X(sim_moe_layer) X(sim_ops_last_error)
struct {
#define X(name) decltype(&::name) name;
    SIM_OPS_CALLS(X)
#undef X
} g;

struct Refused {
    int status;
    std::string why;
};
struct Raised {};  // a Python error is set

void need(bool ok, const char *why) {
    if (!ok) throw Refused{SIM_ERR_INVALID_ARG, why};
}
void need(bool ok, const char *what, const char *why) {
    if (!ok) throw Refused{SIM_ERR_INVALID_ARG, std::string(what) + why};
}

const Tensor &tensor(PyObject *o, const char *what) {
    need(THPVariable_Check(o), what, " must be a tensor");
    return THPVariable_Unpack(o);
}
bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v;
}
int64_t whole(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}

int type_of(at::ScalarType t) {
    return t == at::kFloat ? SIM_TYPE_F32 : t == at::kHalf ? SIM_TYPE_F16 : t == at::kBFloat16 ? SIM_TYPE_BF16 : -1;
}
at::ScalarType dtype(PyObject *o) {
    need(THPDtype_Check(o) && type_of(((THPDtype *)o)->scalar_type) >= 0, "dtype must be float32, float16 or bfloat16");
    return ((THPDtype *)o)->scalar_type;
}

// A matrix whose rows are contiguous.
struct Rows {
    void *p;
    int type;
    int64_t rows, cols, stride;
    c10::Device dev;
};
Rows rows_of(const Tensor &x, const char *what) {
    need(x.dim() == 2, what, " must have two dimensions");
    const int type = type_of(x.scalar_type());
    need(type >= 0, what, " must be float32, float16 or bfloat16");
    need(x.is_cuda(), what, " must be on the GPU");
    const int64_t rows = x.size(0), cols = x.size(1), stride = x.stride(0);
    need((x.stride(1) == 1 || cols <= 1) && (stride >= cols || rows <= 1), what, "'s rows must be contiguous and must not overlap");
    return {x.data_ptr(), type, rows, cols, std::max(stride, cols), x.device()};
}
Rows rows_of(PyObject *o, const char *what) { return rows_of(tensor(o, what), what); }

// A 4-bit tensor whose arrays are as they must be.
struct Stored {
    uint8_t *codes, *scales;
    c10::SmallVector<int64_t, 4> shape;
    int64_t rows, cols;
    c10::Device dev;
};
bool is_mx4(PyObject *o) { return PyObject_TypeCheck(o, (PyTypeObject *)g_mx4); }
Stored stored(PyObject *o, const char *what) {
    need(is_mx4(o), what, " must be in 4 bits");
    const Tensor &codes = tensor(PyTuple_GET_ITEM(o, 0), what), &scales = tensor(PyTuple_GET_ITEM(o, 1), what);
    PyObject *shape = PyTuple_GET_ITEM(o, 2);
    need(PyTuple_Check(shape) && PyTuple_GET_SIZE(shape) > 0, what, ": its shape must be a tuple of sizes");
    c10::SmallVector<int64_t, 4> size;
    int64_t rows = 1;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(shape); i++) {
        if (i) need(!__builtin_mul_overflow(rows, size.back(), &rows), what, " is too large");
        size.push_back(whole(PyTuple_GET_ITEM(shape, i)));
        need(size.back() >= 0 && size.back() < (int64_t)1 << 40, what, ": its shape must be a tuple of sizes");
    }
    const int64_t cols = size.back(), groups = (cols + 255) / 256;
    const auto fits = [&](const Tensor &t, int64_t pitch) {
        return t.dim() == 2 && t.size(0) == rows && t.size(1) == pitch && t.scalar_type() == at::kByte && t.is_contiguous();
    };
    if (!fits(codes, groups * 128) || !fits(scales, groups * 8) || !codes.is_cuda() || scales.device() != codes.device())
        throw Refused{SIM_ERR_INVALID_ARG, std::string("codes and scales of ") + what + " must be contiguous uint8 [" +
                                               std::to_string(rows) + ", " + std::to_string(groups * 128) + "] and [" +
                                               std::to_string(rows) + ", " + std::to_string(groups * 8) + "] on one GPU"};
    return {(uint8_t *)codes.data_ptr(), (uint8_t *)scales.data_ptr(), std::move(size), rows, cols, codes.device()};
}

Tensor fresh(at::IntArrayRef size, at::ScalarType t, c10::Device dev) {
    return at::empty(size, at::TensorOptions(t).device(dev));
}
// A workspace, its address and its size as the calls take them.
struct Space {
    Tensor t;
    void *p = nullptr;
    size_t n;
    Space(size_t bytes, c10::Device dev) : n(bytes) {
        if (n) t = fresh({(int64_t)n}, at::kByte, dev), p = t.data_ptr();
    }
};

// fn(current stream of dev, args...) with that GPU current.
template <typename Fn, typename... A> void call(c10::Device dev, Fn fn, A... args) {
    const c10::DeviceGuard guard(dev);
    const sim_status st = fn((void *)c10::hip::getCurrentHIPStream(dev.index()).stream(), args...);
    if (st != SIM_OK) throw Refused{st, g.sim_ops_last_error()};
}

// A named tuple of n values, which it takes over.
PyObject *named(PyObject *type, std::initializer_list<PyObject *> items) {
    PyObject *r = ((PyTypeObject *)type)->tp_alloc((PyTypeObject *)type, (Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    bool ok = r;
    for (PyObject *o : items) ok = ok && o;
    for (PyObject *o : items) {
        if (ok) PyTuple_SET_ITEM(r, i++, o);
        else Py_XDECREF(o);
    }
    if (!ok) {
        Py_XDECREF(r);
        throw Raised();
    }
    return r;
}
PyObject *sizes(at::IntArrayRef s) {
    PyObject *r = PyTuple_New((Py_ssize_t)s.size());
    if (!r) throw Raised();
    for (size_t i = 0; i < s.size(); i++) PyTuple_SET_ITEM(r, (Py_ssize_t)i, PyLong_FromLongLong(s[i]));
    return r;
}
PyObject *wrap(const Tensor &t) { return THPVariable_Wrap(t); }

// ------------------------------------------------------------------ 4-bit tensors

PyObject *quantize(PyObject *const *a) {  // x, transpose
    const Tensor &x = tensor(a[0], "x");
    const bool transpose = truth(a[1]);
    Tensor flat;
    if (x.dim() != 2) {
        need(x.dim() > 0 && !transpose, "x needs a dimension, and two to be transposed");
        int64_t rows = 1;
        for (int64_t i = 0; i + 1 < x.dim(); i++) rows *= x.size(i);
        flat = x.reshape({rows, x.size(-1)});
    }
    const Rows r = rows_of(flat.defined() ? flat : x, "x");
    const int64_t R = transpose ? r.cols : r.rows, K = transpose ? r.rows : r.cols, groups = (K + 255) / 256;
    const Tensor codes = fresh({R, groups * 128}, at::kByte, r.dev), scales = fresh({R, groups * 8}, at::kByte, r.dev);
    call(r.dev, g.sim_mx4_quantize, r.p, r.type, r.rows, r.cols, r.stride, transpose, (uint8_t *)codes.data_ptr(),
         (uint8_t *)scales.data_ptr());
    return named(g_mx4, {wrap(codes), wrap(scales), transpose ? sizes({R, K}) : sizes(x.sizes())});
}

PyObject *dequantize(PyObject *const *a) {  // q, dtype
    const Stored q = stored(a[0], "q");
    const at::ScalarType type = dtype(a[1]);
    const Tensor out = fresh(q.shape, type, q.dev);
    call(q.dev, g.sim_mx4_dequantize, q.codes, q.scales, q.rows, q.cols, out.data_ptr(), type_of(type), q.cols);
    return wrap(out);
}

// A result of type [M, N], given or new.  One that is given is written behind
// autograd's back: it must not require a gradient, and written() counts the
// write, so that a gradient that has saved it is refused.
struct Result {
    Tensor t;
    Rows r;
    bool given;
    Result(PyObject *out, int64_t M, int64_t N, at::ScalarType type, c10::Device dev)
        : t(out == Py_None ? fresh({M, N}, type, dev) : tensor(out, "out")), r(rows_of(t, "out")), given(out != Py_None) {
        need(r.rows == M && r.cols == N && r.dev == dev, "out must have the result's sizes and be on the same GPU");
        need(!given || !t.requires_grad() || !c10::GradMode::is_enabled(), "out must not require a gradient: the result has none");
    }
    PyObject *written() const {
        if (given && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        return wrap(t);
    }
};

PyObject *matmul(PyObject *const *a) {  // a, b, dtype, out
    const Stored b = stored(a[1], "b");
    need(b.shape.size() == 2, "b must be a 4-bit matrix");
    const int64_t N = b.rows, K = b.cols;
    const at::ScalarType type = a[3] == Py_None ? dtype(a[2]) : tensor(a[3], "out").scalar_type();
    const char *misfit = "a and b differ in their last axis or their GPU";
    if (is_mx4(a[0])) {
        const Stored x = stored(a[0], "a");
        need(x.shape.size() == 2, "a must be a matrix");
        need(x.cols == K && x.dev == b.dev, misfit);
        const Result y(a[3], x.rows, N, type, b.dev);
        call(b.dev, g.sim_mx4_matmul, x.codes, x.scales, b.codes, b.scales, x.rows, N, K, y.r.p, y.r.type, y.r.stride);
        return y.written();
    }
    const Rows x = rows_of(a[0], "a");
    need(x.cols == K && x.dev == b.dev, misfit);
    const Result y(a[3], x.rows, N, type, b.dev);
    if (y.given && y.t.is_alias_of(THPVariable_Unpack(a[0]))) {
        // out may be a itself: then a is read whole before out is written
        const int64_t groups = (K + 255) / 256;
        const Tensor codes = fresh({x.rows, groups * 128}, at::kByte, b.dev), scales = fresh({x.rows, groups * 8}, at::kByte, b.dev);
        uint8_t *const ac = (uint8_t *)codes.data_ptr(), *const as = (uint8_t *)scales.data_ptr();
        call(b.dev, g.sim_mx4_quantize, x.p, x.type, x.rows, K, x.stride, 0, ac, as);
        call(b.dev, g.sim_mx4_matmul, ac, as, b.codes, b.scales, x.rows, N, K, y.r.p, y.r.type, y.r.stride);
        return y.written();
    }
    const Space ws(g.sim_mx4_linear_workspace(x.rows, N, K), b.dev);
    call(b.dev, g.sim_mx4_linear, x.p, x.type, x.stride, b.codes, b.scales, x.rows, N, K, y.r.p, y.r.type, y.r.stride, ws.p, ws.n);
    return y.written();
}

PyObject *linear_grad(PyObject *const *a) {  // dy, x, w, which are wanted: of x, of w
    const Rows dy = rows_of(a[0], "dy"), x = rows_of(a[1], "x"), w = rows_of(a[2], "w");
    const bool want_x = truth(a[3]), want_w = truth(a[4]);
    const int64_t M = dy.rows, N = dy.cols, K = x.cols;
    need(x.rows == M && w.rows == N && w.cols == K && x.dev == dy.dev && w.dev == dy.dev, "dy, x and w do not fit together");
    need(dy.type == x.type && dy.type == w.type, "dy, x and w must have one type");
    const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
    Tensor dx, dw;
    if (want_x) dx = fresh({M, K}, type, dy.dev);
    if (want_w) dw = fresh({N, K}, type, dy.dev);
    const Space ws(g.sim_mx4_linear_grad_workspace(M, N, K), dy.dev);
    call(dy.dev, g.sim_mx4_linear_grad, dy.type, dy.p, dy.stride, x.p, x.stride, w.p, w.stride, M, N, K,
         want_x ? dx.data_ptr() : nullptr, K, want_w ? dw.data_ptr() : nullptr, K, ws.p, ws.n);
    PyObject *px = wrap(dx), *pw = wrap(dw);  // None where there is none
    PyObject *both = PyTuple_Pack(2, px, pw);
    Py_XDECREF(px);
    Py_XDECREF(pw);
    return both;
}

// ------------------------------------------------------------------ router and experts

struct Router {
    Rows z;
    int64_t T, k;
    int32_t E;
    const uint8_t *mask = nullptr;
    int64_t mask_stride = 0;
    Router(PyObject *logits, int64_t k_, PyObject *m) : z(rows_of(logits, "logits")), T(z.rows), k(k_) {
        need(1 <= k && k <= z.cols && k <= SIM_MOE_MAX_TOPK, "k out of range");
        need(z.cols <= SIM_MOE_MAX_EXPERTS, "expert count out of range");
        E = (int32_t)z.cols;
        if (m == Py_None) return;
        const Tensor &t = tensor(m, "mask");
        need((t.scalar_type() == at::kBool || t.scalar_type() == at::kByte) && t.device() == z.dev,
             "mask must be bool or uint8 on the same GPU");
        need((t.dim() == 1 && t.size(0) == E) || (t.dim() == 2 && t.size(0) == T && t.size(1) == E), "mask must be [E] or [T, E]");
        need(E == 1 || t.stride(-1) == 1, "mask must have contiguous rows");
        if (t.dim() == 2) {
            mask_stride = t.stride(0);  // 0 where one row is expanded over the tokens
            need(T <= 1 || mask_stride == 0 || mask_stride >= E, "the rows of mask must not overlap");
        }
        mask = (const uint8_t *)t.data_ptr();
    }
};

PyObject *route(PyObject *const *a) {  // logits, k, mask, renormalize
    const Router r(a[0], whole(a[1]), a[2]);
    const bool renorm = truth(a[3]);
    const Tensor experts = fresh({r.T, r.k}, at::kInt, r.z.dev), weights = fresh({r.T, r.k}, at::kFloat, r.z.dev);
    const Tensor offsets = fresh({r.E + 1}, at::kInt, r.z.dev), order = fresh({r.T * r.k}, at::kInt, r.z.dev);
    const Space ws(g.sim_moe_route_workspace(r.T, r.E, (int32_t)r.k), r.z.dev);
    call(r.z.dev, g.sim_moe_route, r.z.p, r.z.type, r.T, r.E, r.z.stride, r.mask, r.mask_stride, (int32_t)r.k, renorm,
         (int32_t *)experts.data_ptr(), (float *)weights.data_ptr(), (int32_t *)offsets.data_ptr(),
         r.T ? (int32_t *)order.data_ptr() : nullptr, ws.p, ws.n);
    return named(g_routes, {wrap(experts), wrap(weights), wrap(offsets), wrap(order)});
}

PyObject *route_grad(PyObject *const *a) {  // logits, experts, d_weights, mask, renormalize
    const Tensor &e = tensor(a[1], "experts"), &dw = tensor(a[2], "d_weights");
    need(e.dim() == 2, "experts must be [T, k]");
    const Router r(a[0], e.size(1), a[3]);
    const bool renorm = truth(a[4]);
    need(e.size(0) == r.T && dw.sizes() == e.sizes(), "experts and d_weights must be [T, k]");
    need(e.scalar_type() == at::kInt && dw.scalar_type() == at::kFloat, "experts must be int32, d_weights float32");
    need(e.is_contiguous() && dw.is_contiguous(), "experts and d_weights must be contiguous");
    need(e.device() == r.z.dev && dw.device() == r.z.dev, "tensors are on different GPUs");
    const Tensor dz = fresh({r.T, r.E}, THPVariable_Unpack(a[0]).scalar_type(), r.z.dev);
    call(r.z.dev, g.sim_moe_route_grad, r.z.p, r.z.type, r.T, r.E, r.z.stride, r.mask, r.mask_stride, (int32_t)r.k, renorm,
         (const int32_t *)e.data_ptr(), (const float *)dw.data_ptr(), dz.data_ptr());
    return wrap(dz);
}

// The weights of all experts, [E, rows, cols] of type or in 4 bits.
struct Weights {
    const void *p;
    const uint8_t *scales = nullptr;
    int type;
    c10::SmallVector<int64_t, 4> shape;
    Weights(PyObject *o, at::ScalarType x_type, c10::Device dev, const char *what) {
        if (is_mx4(o)) {
            const Stored q = stored(o, what);
            p = q.codes, scales = q.scales, type = SIM_TYPE_MX4, shape = q.shape;
            need(q.dev == dev, "tensors are on different GPUs");
            return;
        }
        const Tensor &t = tensor(o, what);
        need(t.scalar_type() == x_type, "the weights must have the type of x or be in 4 bits");
        need(t.is_contiguous(), "the weights must be contiguous");
        need(t.device() == dev, "tensors are on different GPUs");
        p = t.data_ptr(), type = type_of(x_type), shape.assign(t.sizes().begin(), t.sizes().end());
    }
};

PyObject *layer(PyObject *const *a) {  // x, logits, w13, w2, k, mask, renormalize, out
    const Rows x = rows_of(a[0], "x");
    need(x.type != SIM_TYPE_F32, "x must be float16 or bfloat16");
    const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
    const Router r(a[1], whole(a[4]), a[5]);
    const bool renorm = truth(a[6]);
    need(r.T == x.rows && r.z.dev == x.dev, "x and logits differ in their tokens or their GPU");
    const Weights w13(a[2], type, x.dev, "w13"), w2(a[3], type, x.dev, "w2");
    const int64_t D = x.cols;
    need(w13.type == w2.type && w13.shape.size() == 3 && w2.shape.size() == 3 && w2.shape[0] == r.E && w2.shape[1] == D &&
             w13.shape[0] == r.E && w13.shape[1] == 2 * w2.shape[2] && w13.shape[2] == D,
         "w13 must be [E, 2F, D], w2 [E, D, F], of one kind");
    const int64_t F = w2.shape[2];
    const Result y(a[7], r.T, D, type, x.dev);
    need(y.r.type == x.type, "out must have the type of x");
    const Space ws(g.sim_moe_layer_workspace(r.T, D, r.E, (int32_t)r.k, F), x.dev);
    call(x.dev, g.sim_moe_layer, x.p, x.type, r.T, D, x.stride, r.z.p, r.z.type, r.E, r.z.stride, r.mask, r.mask_stride,
         (int32_t)r.k, renorm, w13.p, w13.scales, w2.p, w2.scales, w2.type, F, y.r.p, y.r.stride, ws.p, ws.n);
    return y.written();
}

// ------------------------------------------------------------------ the module

template <PyObject *(*F)(PyObject *const *), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N || !g_error) {
        PyErr_SetString(PyExc_TypeError, g_error ? "wrong number of arguments" : "setup has not been called");
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Refused &r) {
        if (PyObject *e = PyObject_CallFunction(g_error, "is", r.status, r.why.c_str())) {
            PyErr_SetObject(g_error, e);
            Py_DECREF(e);
        }
    } catch (const Raised &) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}

// SimError, Mx4, Routes, {name: address} of the library's functions
PyObject *setup(PyObject *, PyObject *args) {
    PyObject *error, *mx4, *routes, *at;
    if (!PyArg_ParseTuple(args, "OO!O!O!", &error, &PyType_Type, &mx4, &PyType_Type, &routes, &PyDict_Type, &at)) return nullptr;
#define X(name)                                                                        \
    {                                                                                  \
        PyObject *p = PyDict_GetItemString(at, #name);                                 \
        if (!p) return PyErr_Format(PyExc_KeyError, "%s", #name);                      \
        if (!(g.name = (decltype(&::name))PyLong_AsVoidPtr(p))) return nullptr;        \
    }
    SIM_OPS_CALLS(X)
#undef X
    Py_INCREF(error), Py_INCREF(mx4), Py_INCREF(routes);
    g_mx4 = mx4, g_routes = routes, g_error = error;
    Py_RETURN_NONE;
}

#define ENTRY(name, f, n) {name, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, nullptr},
                         ENTRY("quantize", quantize, 2),
                         ENTRY("dequantize", dequantize, 2),
                         ENTRY("matmul", matmul, 4),
                         ENTRY("linear_grad", linear_grad, 5),
                         ENTRY("route", route, 4),
                         ENTRY("route_grad", route_grad, 5),
                         ENTRY("layer", layer, 8),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_torch(void) { return PyModule_Create(&module); }
