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
#include <cmath>
#include <string>

#include "simgpu_ops.h"

namespace {

using at::Tensor;

PyObject *g_error, *g_mx4, *g_routes, *g_cache;  // SimError, Mx4, Routes, PagedCache

// The library's functions, as it was loaded for the rest of the package.
#define SIM_OPS_CALLS(X)                                                                                            \
    X(sim_mx4_quantize) X(sim_mx4_dequantize) X(sim_mx4_matmul) X(sim_mx4_linear_workspace) X(sim_mx4_linear)       \
        X(sim_mx4_linear_grad_workspace) X(sim_mx4_linear_grad) X(sim_moe_route_workspace) X(sim_moe_route)         \
            X(sim_moe_route_grad) X(sim_moe_route_scored) X(sim_moe_route_scored_grad) X(sim_moe_layer_workspace)       \
                X(sim_moe_layer) X(sim_moe_experts_workspace) X(sim_moe_experts) X(sim_cache_append) X(sim_cache_attention_workspace) X(sim_cache_attention) X(sim_sample_workspace) X(sim_sample) X(sim_ops_last_error)
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

int score_of(PyObject *o) {
    const char *s = PyUnicode_Check(o) ? PyUnicode_AsUTF8(o) : nullptr;
    const std::string name = s ? s : "";
    need(name == "softmax" || name == "sigmoid", "score must be \"softmax\" or \"sigmoid\"");
    return name == "softmax" ? SIM_SCORE_SOFTMAX : SIM_SCORE_SIGMOID;
}
double number(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    return v;
}
int32_t small(PyObject *o, const char *what) {
    const int64_t v = whole(o);
    need(v > INT32_MIN && v < INT32_MAX, what, " out of range");
    return (int32_t)v;
}

PyObject *route(PyObject *const *a) {  // logits, k, mask, renormalize, score, bias, groups, top_groups, group_best, scale
    const Router r(a[0], whole(a[1]), a[2]);
    const bool renorm = truth(a[3]);
    const int score = score_of(a[4]);
    const float *bias = nullptr;
    if (a[5] != Py_None) {
        const Tensor &t = tensor(a[5], "bias");
        need(t.dim() == 1 && t.size(0) == r.E && t.scalar_type() == at::kFloat && t.is_contiguous() && t.device() == r.z.dev,
             "bias must be contiguous float32 [E] on the same GPU");
        bias = (const float *)t.data_ptr();
    }
    const int32_t groups = small(a[6], "groups"), top_groups = a[7] == Py_None ? groups : small(a[7], "top_groups"), best = small(a[8], "group_best");
    const float scale = (float)number(a[9]);
    const bool plain = score == SIM_SCORE_SOFTMAX && !bias && groups == 1 && top_groups == 1 && (best == 1 || best == 2) && scale == 1.f;
    const Tensor experts = fresh({r.T, r.k}, at::kInt, r.z.dev), weights = fresh({r.T, r.k}, at::kFloat, r.z.dev);
    const Tensor offsets = fresh({r.E + 1}, at::kInt, r.z.dev), order = fresh({r.T * r.k}, at::kInt, r.z.dev);
    const Space ws(g.sim_moe_route_workspace(r.T, r.E, (int32_t)r.k), r.z.dev);
    int32_t *const e = (int32_t *)experts.data_ptr(), *const o = (int32_t *)offsets.data_ptr(), *const s = r.T ? (int32_t *)order.data_ptr() : nullptr;
    float *const w = (float *)weights.data_ptr();
    if (plain)
        call(r.z.dev, g.sim_moe_route, r.z.p, r.z.type, r.T, r.E, r.z.stride, r.mask, r.mask_stride, (int32_t)r.k, renorm, e, w, o, s, ws.p, ws.n);
    else
        call(r.z.dev, g.sim_moe_route_scored, r.z.p, r.z.type, r.T, r.E, r.z.stride, r.mask, r.mask_stride, score, bias, groups, top_groups,
             best, (int32_t)r.k, renorm, scale, e, w, o, s, ws.p, ws.n);
    return named(g_routes, {wrap(experts), wrap(weights), wrap(offsets), wrap(order)});
}

PyObject *route_grad(PyObject *const *a) {  // logits, experts, d_weights, mask, renormalize, score, scale
    const Tensor &e = tensor(a[1], "experts"), &dw = tensor(a[2], "d_weights");
    need(e.dim() == 2, "experts must be [T, k]");
    const Router r(a[0], e.size(1), a[3]);
    const bool renorm = truth(a[4]);
    need(e.size(0) == r.T && dw.sizes() == e.sizes(), "experts and d_weights must be [T, k]");
    need(e.scalar_type() == at::kInt && dw.scalar_type() == at::kFloat, "experts must be int32, d_weights float32");
    need(e.is_contiguous() && dw.is_contiguous(), "experts and d_weights must be contiguous");
    need(e.device() == r.z.dev && dw.device() == r.z.dev, "tensors are on different GPUs");
    const Tensor dz = fresh({r.T, r.E}, THPVariable_Unpack(a[0]).scalar_type(), r.z.dev);
    call(r.z.dev, g.sim_moe_route_scored_grad, r.z.p, r.z.type, r.T, r.E, r.z.stride, r.mask, r.mask_stride, score_of(a[5]), (int32_t)r.k,
         renorm, (float)number(a[6]), (const int32_t *)e.data_ptr(), (const float *)dw.data_ptr(), dz.data_ptr());
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

PyObject *experts(PyObject *const *a) {  // x, experts, weights, w13, w2, first, out
    const Rows x = rows_of(a[0], "x");
    need(x.type != SIM_TYPE_F32, "x must be float16 or bfloat16");
    const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
    const Tensor &e = tensor(a[1], "experts"), &w = tensor(a[2], "weights");
    need(e.dim() == 2 && e.size(0) == x.rows && w.sizes() == e.sizes(), "experts and weights must be [T, k]");
    need(e.scalar_type() == at::kInt && w.scalar_type() == at::kFloat, "experts must be int32, weights float32");
    need(e.is_contiguous() && w.is_contiguous(), "experts and weights must be contiguous");
    need(e.device() == x.dev && w.device() == x.dev, "tensors are on different GPUs");
    const int64_t k = e.size(1), D = x.cols;
    need(k >= 1 && k <= SIM_MOE_MAX_TOPK, "k out of range");
    const Weights w13(a[3], type, x.dev, "w13"), w2(a[4], type, x.dev, "w2");
    need(w13.type == w2.type && w13.shape.size() == 3 && w2.shape.size() == 3 && w2.shape[1] == D && w13.shape[0] == w2.shape[0] &&
             w13.shape[1] == 2 * w2.shape[2] && w13.shape[2] == D,
         "w13 must be [n, 2F, D], w2 [n, D, F], of one kind");
    const int64_t n = w2.shape[0], F = w2.shape[2];
    need(n >= 1 && n <= SIM_MOE_MAX_EXPERTS, "expert count out of range");
    const int32_t first = small(a[5], "first");
    const Result y(a[6], x.rows, D, type, x.dev);
    need(y.r.type == x.type, "out must have the type of x");
    const Space ws(g.sim_moe_experts_workspace(x.rows, D, (int32_t)n, (int32_t)k, F), x.dev);
    call(x.dev, g.sim_moe_experts, x.p, x.type, x.rows, D, x.stride, (const int32_t *)e.data_ptr(), (const float *)w.data_ptr(), (int32_t)k,
         first, (int32_t)n, w13.p, w13.scales, w2.p, w2.scales, w2.type, F, y.r.p, y.r.stride, ws.p, ws.n);
    return y.written();
}

// ------------------------------------------------------------------ paged cache

// A tensor [N, heads, D] whose rows of D are contiguous, for reading.
struct Heads {
    const void *p;
    at::ScalarType type;
    int64_t n, heads, D, stride, head_stride;
    c10::Device dev;
};
Heads heads_of(const Tensor &x, const char *what) {
    need(x.dim() == 3, what, " must have three dimensions");
    need(x.scalar_type() == at::kHalf || x.scalar_type() == at::kBFloat16, what, " must be float16 or bfloat16");
    need(x.is_cuda(), what, " must be on the GPU");
    need(x.stride(2) == 1 || x.size(2) <= 1, what, "'s rows must be contiguous");
    return {x.data_ptr(), x.scalar_type(), x.size(0), x.size(1), x.size(2), x.size(0) > 1 ? x.stride(0) : 0, x.size(1) > 1 ? x.stride(1) : 0, x.device()};
}
Heads heads_of(PyObject *o, const char *what) { return heads_of(tensor(o, what), what); }

struct Paged {
    void *k, *v;
    at::ScalarType type;
    int64_t pages, heads, size, D, k_stride, v_stride;
    c10::Device dev;
};
Paged paged(PyObject *o) {
    need(PyObject_TypeCheck(o, (PyTypeObject *)g_cache), "cache must be a PagedCache");
    const Tensor &k = tensor(PyTuple_GET_ITEM(o, 0), "cache.k"), &v = tensor(PyTuple_GET_ITEM(o, 1), "cache.v");
    need(k.dim() == 4 && v.dim() == 4 && k.sizes() == v.sizes(), "cache.k and cache.v must be [pages, kv heads, page size, D]");
    need(k.scalar_type() == v.scalar_type() && (k.scalar_type() == at::kHalf || k.scalar_type() == at::kBFloat16),
         "the cache must be float16 or bfloat16");
    need(k.is_cuda() && v.device() == k.device(), "the cache must be on one GPU");
    const int64_t pages = k.size(0), heads = k.size(1), size = k.size(2), D = k.size(3);
    need(heads > 0 && heads < 1 << 20 && size > 0 && size < (int64_t)1 << 31, "bad sizes of the cache");
    need(D > 0 && D <= SIM_CACHE_MAX_D, "D must be a multiple of 8 up to 256");
    const auto whole_pages = [&](const Tensor &t) {
        return (D <= 1 || t.stride(3) == 1) && (size == 1 || t.stride(2) == D) && (heads == 1 || t.stride(1) == size * D);
    };
    need(whole_pages(k) && whole_pages(v), "the cache's pages must be contiguous");
    const int64_t page = heads * size * D;
    return {k.data_ptr(), v.data_ptr(), k.scalar_type(), pages, heads, size, D, pages > 1 ? k.stride(0) : page, pages > 1 ? v.stride(0) : page, k.device()};
}

PyObject *append(PyObject *const *a) {  // cache, k, v, slots
    const Paged c = paged(a[0]);
    const Heads k = heads_of(a[1], "k"), v = heads_of(a[2], "v");
    const Tensor &slots = tensor(a[3], "slots");
    need(k.n == v.n && k.heads == c.heads && v.heads == c.heads && k.D == c.D && v.D == c.D, "k and v must be [T, kv heads, D]");
    need(k.type == c.type && v.type == c.type, "k and v must have the cache's type");
    need(slots.dim() == 1 && slots.size(0) == k.n && slots.scalar_type() == at::kLong && slots.is_contiguous(), "slots must be contiguous int64 [T]");
    need(k.dev == c.dev && v.dev == c.dev && slots.device() == c.dev, "tensors are on different GPUs");
    for (int i = 0; i < 2; i++)
        need(!c10::GradMode::is_enabled() || !THPVariable_Unpack(PyTuple_GET_ITEM(a[0], i)).requires_grad(),
             "the cache must not require a gradient: it is written in place");
    call(c.dev, g.sim_cache_append, type_of(c.type), k.p, k.stride, k.head_stride, v.p, v.stride, v.head_stride, k.n, (int32_t)c.heads,
         (int32_t)c.D, (const int64_t *)slots.data_ptr(), c.k, c.k_stride, c.v, c.v_stride, c.pages, (int32_t)c.size);
    for (int i = 0; i < 2; i++) {
        const Tensor &t = THPVariable_Unpack(PyTuple_GET_ITEM(a[0], i));
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
    Py_RETURN_NONE;
}

PyObject *attention(PyObject *const *a) {  // q, cache, table, lengths, scale, window, return_lse, out
    const Heads q = heads_of(a[0], "q");
    const Paged c = paged(a[1]);
    const Tensor &table = tensor(a[2], "table"), &lengths = tensor(a[3], "lengths");
    need(q.D == c.D, "q must be [B, q heads, D]");
    need(q.heads > 0 && q.heads < 1 << 20 && q.heads % c.heads == 0, "the cache's heads must divide q's");
    need(q.type == c.type, "q must have the cache's type");
    need(table.dim() == 2 && table.size(0) == q.n && table.scalar_type() == at::kInt && (table.size(1) <= 1 || table.stride(1) == 1) && table.size(1) < (int64_t)1 << 31,
         "table must be int32 [B, pages] with contiguous rows");
    need(lengths.dim() == 1 && lengths.size(0) == q.n && lengths.scalar_type() == at::kInt && lengths.is_contiguous(), "lengths must be contiguous int32 [B]");
    need(q.dev == c.dev && table.device() == c.dev && lengths.device() == c.dev, "tensors are on different GPUs");
    const int64_t window = whole(a[5]);
    need(window >= 0 && window < (int64_t)1 << 31, "window must not be negative");
    const bool want_lse = truth(a[6]);
    const double scale = a[4] == Py_None ? 1 / std::sqrt((double)c.D) : number(a[4]);
    Tensor out, lse;
    const bool given = a[7] != Py_None;
    if (given) {
        out = tensor(a[7], "out");
        const Heads o = heads_of(out, "out");
        need(o.n == q.n && o.heads == q.heads && o.D == q.D && o.type == q.type && o.dev == q.dev, "out must be as q");
        need((o.heads == 1 || o.head_stride == o.D) && (o.n <= 1 || o.stride >= o.heads * o.D), "out's heads must be contiguous and must not overlap");
        need(!out.requires_grad() || !c10::GradMode::is_enabled(), "out must not require a gradient: the result has none");
        for (PyObject *o : {(PyObject *)a[0], PyTuple_GET_ITEM(a[1], 0), PyTuple_GET_ITEM(a[1], 1)})
            need(!out.is_alias_of(THPVariable_Unpack(o)), "out must not share memory with q or the cache");
    } else {
        out = fresh({q.n, q.heads, q.D}, q.type, q.dev);
    }
    if (want_lse) lse = fresh({q.n, q.heads}, at::kFloat, q.dev);
    const Space ws(g.sim_cache_attention_workspace(q.n, (int32_t)q.heads, (int32_t)c.heads, (int32_t)c.D, (int32_t)table.size(1), (int32_t)c.size, (int32_t)window), c.dev);
    call(c.dev, g.sim_cache_attention, type_of(q.type), q.p, q.stride, q.head_stride, q.n, (int32_t)q.heads, (int32_t)c.heads, (int32_t)c.D, c.k,
         c.k_stride, c.v, c.v_stride, c.pages, (int32_t)c.size, (const int32_t *)table.data_ptr(), table.size(0) > 1 ? table.stride(0) : 0,
         (int32_t)table.size(1), (const int32_t *)lengths.data_ptr(), (float)scale, (int32_t)window, out.data_ptr(),
         out.size(0) > 1 ? out.stride(0) : q.heads * q.D, want_lse ? (float *)lse.data_ptr() : nullptr, ws.p, ws.n);
    if (given && !out.is_inference()) out.unsafeGetTensorImpl()->bump_version();
    if (!want_lse) return wrap(out);
    PyObject *po = wrap(out), *pl = wrap(lse);
    PyObject *both = po && pl ? PyTuple_Pack(2, po, pl) : nullptr;
    Py_XDECREF(po);
    Py_XDECREF(pl);
    return both;
}

// ------------------------------------------------------------------ the next token

// A parameter of every row, or one number for all.
template <typename V> struct Setting {
    const V *p = nullptr;
    V all = 0;
    Setting(PyObject *o, int64_t B, c10::Device dev, const char *what) {
        constexpr bool whole_number = std::is_integral<V>::value;
        if (THPVariable_Check(o)) {
            const Tensor &t = THPVariable_Unpack(o);
            need(t.dim() == 1 && t.size(0) == B && t.scalar_type() == (whole_number ? at::kInt : at::kFloat) && t.is_contiguous() && t.device() == dev,
                 what, whole_number ? " must be a number or contiguous int32 [B] on the same GPU" : " must be a number or contiguous float32 [B] on the same GPU");
            if (B) p = (const V *)t.data_ptr();
        } else {
            if constexpr (whole_number) all = small(o, what);
            else all = (V)number(o);
        }
    }
};

PyObject *sample(PyObject *const *a) {  // logits, u, temperature, top_k, top_p, min_p
    const Rows z = rows_of(a[0], "logits");
    need(z.cols >= 1 && z.cols < (int64_t)1 << 31, "there must be a logit to choose");
    const Tensor &u = tensor(a[1], "u");
    need(u.dim() == 1 && u.size(0) == z.rows && u.scalar_type() == at::kFloat && u.is_contiguous() && u.device() == z.dev,
         "u must be contiguous float32 [B] on the same GPU");
    const Setting<float> t(a[2], z.rows, z.dev, "temperature"), p(a[4], z.rows, z.dev, "top_p"), m(a[5], z.rows, z.dev, "min_p");
    const Setting<int32_t> k(a[3], z.rows, z.dev, "top_k");
    const Tensor tokens = fresh({z.rows}, at::kInt, z.dev);
    const Space ws(g.sim_sample_workspace(z.rows, (int32_t)z.cols), z.dev);
    call(z.dev, g.sim_sample, z.p, z.type, z.rows, (int32_t)z.cols, z.stride, (const float *)u.data_ptr(), t.p, t.all, k.p, k.all, p.p, p.all, m.p,
         m.all, (int32_t *)tokens.data_ptr(), ws.p, ws.n);
    return wrap(tokens);
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

// SimError, Mx4, Routes, PagedCache, {name: address} of the library's functions
PyObject *setup(PyObject *, PyObject *args) {
    PyObject *error, *mx4, *routes, *cache, *at;
    if (!PyArg_ParseTuple(args, "OO!O!O!O!", &error, &PyType_Type, &mx4, &PyType_Type, &routes, &PyType_Type, &cache, &PyDict_Type, &at))
        return nullptr;
#define X(name)                                                                        \
    {                                                                                  \
        PyObject *p = PyDict_GetItemString(at, #name);                                 \
        if (!p) return PyErr_Format(PyExc_KeyError, "%s", #name);                      \
        if (!(g.name = (decltype(&::name))PyLong_AsVoidPtr(p))) return nullptr;        \
    }
    SIM_OPS_CALLS(X)
#undef X
    Py_INCREF(error), Py_INCREF(mx4), Py_INCREF(routes), Py_INCREF(cache);
    g_mx4 = mx4, g_routes = routes, g_cache = cache, g_error = error;
    Py_RETURN_NONE;
}

#define ENTRY(name, f, n) {name, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, nullptr},
                         ENTRY("quantize", quantize, 2),
                         ENTRY("dequantize", dequantize, 2),
                         ENTRY("matmul", matmul, 4),
                         ENTRY("linear_grad", linear_grad, 5),
                         ENTRY("route", route, 10),
                         ENTRY("route_grad", route_grad, 7),
                         ENTRY("layer", layer, 8),
                         ENTRY("experts", experts, 7),
                         ENTRY("sample", sample, 6),
                         ENTRY("append", append, 4),
                         ENTRY("attention", attention, 8),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ops_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ops_torch(void) { return PyModule_Create(&module); }
