"""Operators of an expert-parallel step on the GPU, next to the traffic that
``sim`` simulates: 4-bit microscaled tensors (what travels, and the products of
linear layers), the router with the experts' token lists (who gets it), and
the experts' layer for few tokens (what is computed there).

Functions marshal torch tensors for the C ABI of ``include/simgpu_ops.h``
(there the layouts, formulas and limits are stated).  Work is enqueued on the
current stream of the tensors' device; results and workspaces come from
torch's allocator, so a call may be captured into a graph.  Every step runs in
the library's HIP kernels; there is no host or torch fallback.  Refused
arguments raise ``SimError`` before anything is enqueued.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

import torch

from . import sim
from .sim import SIM_ERR_INVALID_ARG, SIM_OK, SimError

EXPORTS = ("sim_mx4_code_pitch", "sim_mx4_scale_pitch", "sim_mx4_quantize", "sim_mx4_dequantize",
           "sim_mx4_matmul_workspace", "sim_mx4_matmul", "sim_mx4_linear_workspace", "sim_mx4_linear",
           "sim_moe_route_workspace", "sim_moe_route", "sim_moe_route_grad", "sim_moe_layer_workspace",
           "sim_moe_layer", "sim_ops_last_error")

MAX_EXPERTS, MAX_TOPK, MAX_LAYER_TOKENS = 1024, 32, 1024
_TYPE = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_MX4 = 3

_lib = None


def lib():
    """libsimgpu.so with the operators' signatures."""
    global _lib
    if _lib is None:
        L = sim.lib()
        P, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.sim_mx4_code_pitch.argtypes = L.sim_mx4_scale_pitch.argtypes = [i64]
        L.sim_mx4_code_pitch.restype = L.sim_mx4_scale_pitch.restype = i64
        L.sim_mx4_quantize.argtypes = [P, P, i32, i64, i64, i64, i32, P, P]
        L.sim_mx4_dequantize.argtypes = [P, P, P, i64, i64, P, i32, i64]
        L.sim_mx4_matmul_workspace.argtypes = L.sim_mx4_linear_workspace.argtypes = [i64, i64, i64]
        L.sim_mx4_matmul_workspace.restype = L.sim_mx4_linear_workspace.restype = sz
        L.sim_mx4_matmul.argtypes = [P, P, P, P, P, i64, i64, i64, P, i32, i64, P, sz]
        L.sim_mx4_linear.argtypes = [P, P, i32, i64, P, P, i64, i64, i64, P, i32, i64, P, sz]
        L.sim_moe_route_workspace.argtypes = [i64, i32, i32]
        L.sim_moe_route_workspace.restype = sz
        L.sim_moe_route.argtypes = [P, P, i32, i64, i32, i64, P, i64, i32, i32, P, P, P, P, P, sz]
        L.sim_moe_route_grad.argtypes = [P, P, i32, i64, i32, i64, P, i64, i32, i32, P, P, P]
        L.sim_moe_layer_workspace.argtypes = [i64, i64, i32, i32, i64]
        L.sim_moe_layer_workspace.restype = sz
        L.sim_moe_layer.argtypes = [P, P, i32, i64, i64, i64, P, i32, i32, i64, P, i64, i32, i32, P, P, P, P, i32,
                                    i64, P, i64, P, sz]
        for name in ("sim_mx4_quantize", "sim_mx4_dequantize", "sim_mx4_matmul", "sim_mx4_linear", "sim_moe_route",
                     "sim_moe_route_grad", "sim_moe_layer"):
            getattr(L, name).restype = C.c_int
        L.sim_ops_last_error.argtypes = []
        L.sim_ops_last_error.restype = C.c_char_p
        _lib = L
    return _lib


def _call(device, fn, *args):
    """fn(current stream of device, *args) with that device current."""
    if device.index == torch.cuda.current_device():
        st = fn(torch.cuda.current_stream().cuda_stream, *args)
    else:
        with torch.cuda.device(device):
            st = fn(torch.cuda.current_stream().cuda_stream, *args)
    if st != SIM_OK:
        raise SimError(st, lib().sim_ops_last_error().decode())


def _need(ok, why):
    if not ok:
        raise SimError(SIM_ERR_INVALID_ARG, why)


def _rows(x, what):
    """A matrix whose rows are contiguous; (pointer, row stride)."""
    _need(x.dim() == 2, f"{what} must have two dimensions")
    _need(x.dtype in _TYPE, f"{what} must be float32, float16 or bfloat16")
    _need(x.is_cuda, f"{what} must be on the GPU")
    _need(x.shape[1] <= 1 or x.stride(1) == 1, f"{what} must have contiguous rows")
    _need(x.shape[0] <= 1 or x.stride(0) >= x.shape[1], f"the rows of {what} must not overlap")
    return x.data_ptr(), max(x.stride(0), x.shape[1])


def _same_device(device, *tensors):
    _need(all(t is None or t.device == device for t in tensors), "tensors are on different devices")


def _space(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _p(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ 4-bit tensors

class Mx4(NamedTuple):
    """A 4-bit microscaled tensor: ``shape`` [..., K] with the leading axes
    flattened to rows in ``codes`` [rows, code pitch] and ``scales`` [rows,
    scale pitch] (uint8)."""
    codes: torch.Tensor
    scales: torch.Tensor
    shape: tuple

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()


def _check_mx4(q, what):
    K = q.shape[-1]
    rows = 1
    for n in q.shape[:-1]:
        rows *= n
    groups = -(-K // 256)
    for t, pitch, name in ((q.codes, groups * 128, "codes"), (q.scales, groups * 8, "scales")):
        _need(t.dtype == torch.uint8 and t.is_cuda and t.is_contiguous() and t.shape == (rows, pitch),
              f"the {name} of {what} must be a contiguous uint8 [{rows}, {pitch}] on the GPU")
    return rows, K


def mx4_quantize(x, transpose=False) -> Mx4:
    """``x`` [..., K] in 4 bits, a scale for 32 elements along its last axis.
    With ``transpose`` (two dimensions) the result is that of ``x.t()``."""
    _need(x.dim() >= 1, "x needs a dimension")
    if transpose:
        _need(x.dim() == 2, "only a matrix can be transposed")
    flat = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
    ptr, stride = _rows(flat, "x")
    rows, cols = flat.shape
    R, K = (cols, rows) if transpose else (rows, cols)
    groups = -(-K // 256)
    codes = torch.empty((R, groups * 128), dtype=torch.uint8, device=x.device)
    scales = torch.empty((R, groups * 8), dtype=torch.uint8, device=x.device)
    _call(x.device, lib().sim_mx4_quantize, ptr, _TYPE[x.dtype], rows, cols, stride, int(transpose), codes.data_ptr(),
          scales.data_ptr())
    return Mx4(codes, scales, (R, K) if transpose else tuple(x.shape))


def mx4_dequantize(q: Mx4, dtype=torch.bfloat16):
    """The values that ``q`` stands for."""
    rows, K = _check_mx4(q, "q")
    _need(dtype in _TYPE, "dtype must be float32, float16 or bfloat16")
    out = torch.empty((rows, K), dtype=dtype, device=q.codes.device)
    _call(out.device, lib().sim_mx4_dequantize, q.codes.data_ptr(), q.scales.data_ptr(), rows, K, out.data_ptr(),
          _TYPE[dtype], K)
    return out if len(q.shape) == 2 else out.view(q.shape)


def mx4_matmul(a, b: Mx4, dtype=torch.bfloat16, out=None):
    """``a @ b.T`` with both in 4 bits along their last axis, summed in 32
    bits.  ``a`` [M, K] is an ``Mx4``, or a plain tensor that is put into 4
    bits on the way; ``b`` [N, K]; the result is [M, N] of ``dtype`` (or of
    ``out``, which may have strided rows)."""
    _need(isinstance(b, Mx4) and len(b.shape) == 2, "b must be a 4-bit matrix")
    N, K = _check_mx4(b, "b")
    plain = not isinstance(a, Mx4)
    if plain:
        ptr, stride = _rows(a, "a")
        M, device = a.shape[0], a.device
    else:
        _need(len(a.shape) == 2, "a must be a matrix")
        M, device = _check_mx4(a, "a")[0], a.codes.device
        _same_device(device, a.scales)
    _need(a.shape[1] == K, "a and b differ in their last axis")
    if out is None:
        _need(dtype in _TYPE, "dtype must be float32, float16 or bfloat16")
        out = torch.empty((M, N), dtype=dtype, device=device)
    _need(tuple(out.shape) == (M, N), "out has the wrong shape")
    optr, ostride = _rows(out, "out")
    _same_device(device, b.codes, b.scales, out)
    L = lib()
    if plain:
        n = L.sim_mx4_linear_workspace(M, N, K)
        ws = _space(n, device)
        _call(device, L.sim_mx4_linear, ptr, _TYPE[a.dtype], stride, b.codes.data_ptr(), b.scales.data_ptr(), M, N, K, optr,
              _TYPE[out.dtype], ostride, _p(ws), n)
    else:
        n = L.sim_mx4_matmul_workspace(M, N, K)
        ws = _space(n, device)
        _call(device, L.sim_mx4_matmul, a.codes.data_ptr(), a.scales.data_ptr(), b.codes.data_ptr(), b.scales.data_ptr(), M,
              N, K, optr, _TYPE[out.dtype], ostride, _p(ws), n)
    return out


def mx4_linear_grad(dy, x, w):
    """Gradients ``(dx, dw)`` of ``y = x @ w.T`` computed in 4 bits, where
    rounding to 4 bits passes gradients through: ``dx = dy @ w`` and ``dw =
    dy.T @ x``, each operand quantised along the axis that is summed over."""
    for t, n in ((dy, "dy"), (x, "x"), (w, "w")):
        _rows(t, n)
    _need(dy.shape == (x.shape[0], w.shape[0]) and x.shape[1] == w.shape[1], "dy, x and w do not fit together")
    _same_device(dy.device, x, w)
    dx = mx4_matmul(dy, mx4_quantize(w, transpose=True), dtype=x.dtype)
    dw = mx4_matmul(mx4_quantize(dy, transpose=True), mx4_quantize(x, transpose=True), dtype=w.dtype)
    return dx, dw


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return mx4_matmul(x, mx4_quantize(w), dtype=x.dtype)

    @staticmethod
    def backward(ctx, dy):
        return mx4_linear_grad(dy.contiguous(), *ctx.saved_tensors)


def mx4_linear(x, w):
    """``x @ w.T`` with both put into 4 bits, for training: x [M, K] and w
    [N, K] get the gradients of ``mx4_linear_grad``."""
    return _Linear.apply(x, w)


# ------------------------------------------------------------------ router and experts

class Routes(NamedTuple):
    """What a router decided for T tokens: ``experts`` [T, k] (int32, -1:
    none) and ``weights`` [T, k] (float32); and the experts' lists: ``order``
    [T k] holds slots (token k + choice) sorted by expert, those of expert e at
    ``offsets[e] .. offsets[e + 1] - 1``."""
    experts: torch.Tensor
    weights: torch.Tensor
    offsets: torch.Tensor
    order: torch.Tensor


def _route_args(logits, k, mask):
    _need(logits.dim() == 2 and 1 <= k <= min(logits.shape[1], MAX_TOPK), "k out of range")
    ptr, stride = _rows(logits, "logits")
    T, E = logits.shape
    mptr, mstride = None, 0
    if mask is not None:
        _need(mask.dtype in (torch.bool, torch.uint8), "mask must be bool or uint8")
        _need(tuple(mask.shape) in ((E,), (T, E)), "mask must be [E] or [T, E]")
        _need(E == 1 or mask.stride(-1) == 1, "mask must have contiguous rows")
        _same_device(logits.device, mask)
        if mask.dim() == 2:
            mstride = mask.stride(0)  # 0 where one row is expanded over the tokens
            _need(T <= 1 or mstride == 0 or mstride >= E, "the rows of mask must not overlap")
        mptr = mask.data_ptr()
    return ptr, _TYPE[logits.dtype], T, E, stride, mptr, mstride, int(k)


def moe_route(logits, k, mask=None, renormalize=True) -> Routes:
    """The k experts of each token with the highest logits [T, E], their
    softmax weights, and the experts' lists of slots.  ``mask`` ([E] or [T,
    E], true = allowed) takes experts out; ``renormalize`` divides a token's
    weights by their sum."""
    args = _route_args(logits, k, mask)
    T, E = logits.shape
    dev = logits.device
    i = torch.empty(2 * T * k + E + 1, dtype=torch.int32, device=dev)
    experts, order, offsets = i[:T * k].view(T, k), i[T * k:2 * T * k], i[2 * T * k:]
    weights = torch.empty((T, k), dtype=torch.float32, device=dev)
    L = lib()
    n = L.sim_moe_route_workspace(T, E, k)
    ws = _space(n, dev)
    _call(dev, L.sim_moe_route, *args, int(renormalize), experts.data_ptr(), weights.data_ptr(), offsets.data_ptr(),
          order.data_ptr(), _p(ws), n)
    return Routes(experts, weights, offsets, order)


def moe_route_grad(logits, experts, d_weights, mask=None, renormalize=True):
    """Gradient of ``moe_route``'s weights with respect to the logits, from
    the gradient [T, k] of the weights."""
    _need(experts.dim() == 2, "experts must be [T, k]")
    T, k = experts.shape
    args = _route_args(logits, k, mask)
    _need(logits.shape[0] == T and tuple(d_weights.shape) == (T, k), "experts and d_weights must be [T, k]")
    _need(experts.dtype == torch.int32 and d_weights.dtype == torch.float32, "experts must be int32, d_weights float32")
    _need(experts.is_contiguous() and d_weights.is_contiguous(), "experts and d_weights must be contiguous")
    _same_device(logits.device, experts, d_weights)
    dz = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    _call(logits.device, lib().sim_moe_route_grad, *args, int(renormalize), experts.data_ptr(), d_weights.data_ptr(),
          dz.data_ptr())
    return dz


class _RouteWeights(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, mask, renormalize):
        r = moe_route(logits, k, mask, renormalize)
        ctx.save_for_backward(logits, r.experts, mask)
        ctx.renormalize = renormalize
        ctx.mark_non_differentiable(r.experts, r.offsets, r.order)
        return r.experts, r.weights, r.offsets, r.order

    @staticmethod
    def backward(ctx, _e, dw, _o, _s):
        logits, experts, mask = ctx.saved_tensors
        return moe_route_grad(logits, experts, dw.contiguous(), mask, ctx.renormalize), None, None, None


def moe_route_train(logits, k, mask=None, renormalize=True) -> Routes:
    """``moe_route`` whose weights carry gradients to the logits."""
    return Routes(*_RouteWeights.apply(logits, k, mask, renormalize))


def moe_layer(x, logits, w13, w2, k, mask=None, renormalize=True, out=None):
    """The experts' layer for few tokens (at most ``MAX_LAYER_TOKENS``): each
    token x [T, D] goes through the k experts that ``moe_route`` gives it,
    ``w2[e] @ (silu(g) * u)`` with ``g, u = w13[e] @ x`` (w13 [E, 2F, D]: F
    gate rows, then F up rows; w2 [E, D, F]), and gets their weighted sum.  x
    is float16 or bfloat16; the weights have its type, or are ``Mx4``."""
    xptr, xstride = _rows(x, "x")
    _need(x.dtype != torch.float32, "x must be float16 or bfloat16")
    args = _route_args(logits, k, mask)
    T, D = x.shape
    E = logits.shape[1]
    _need(logits.shape[0] == T, "x and logits differ in their tokens")
    mx4 = isinstance(w13, Mx4)
    _need(mx4 == isinstance(w2, Mx4), "w13 and w2 must be of one kind")
    _need(len(w13.shape) == 3 and len(w2.shape) == 3, "w13 must be [E, 2F, D], w2 [E, D, F]")
    F = w2.shape[2]
    _need(tuple(w13.shape) == (E, 2 * F, D) and tuple(w2.shape) == (E, D, F), "w13 must be [E, 2F, D], w2 [E, D, F]")
    if mx4:
        _check_mx4(w13, "w13")
        _check_mx4(w2, "w2")
        wargs = (w13.codes.data_ptr(), w13.scales.data_ptr(), w2.codes.data_ptr(), w2.scales.data_ptr(), _MX4)
        _same_device(x.device, logits, w13.codes, w13.scales, w2.codes, w2.scales)
    else:
        _need(w13.dtype == x.dtype and w2.dtype == x.dtype, "the weights must have the type of x or be in 4 bits")
        _need(w13.is_contiguous() and w2.is_contiguous(), "the weights must be contiguous")
        wargs = (w13.data_ptr(), None, w2.data_ptr(), None, _TYPE[x.dtype])
        _same_device(x.device, logits, w13, w2)
    if out is None:
        out = torch.empty((T, D), dtype=x.dtype, device=x.device)
    _need(tuple(out.shape) == (T, D) and out.dtype == x.dtype, "out must be like x")
    optr, ostride = _rows(out, "out")
    _same_device(x.device, out)
    L = lib()
    n = L.sim_moe_layer_workspace(T, D, E, k, F)
    ws = _space(n, x.device)
    _call(x.device, L.sim_moe_layer, xptr, _TYPE[x.dtype], T, D, xstride, *args[:2], args[3], args[4], *args[5:],
          int(renormalize), *wargs, F, optr, ostride, _p(ws), n)
    return out
