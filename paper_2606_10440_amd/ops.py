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
import math
from typing import NamedTuple

import torch

from . import sim
from .sim import SIM_ERR_INVALID_ARG, SIM_OK, SimError

EXPORTS = ("sim_mx4_code_pitch", "sim_mx4_scale_pitch", "sim_mx4_quantize", "sim_mx4_dequantize",
           "sim_mx4_matmul", "sim_mx4_linear_workspace", "sim_mx4_linear",
           "sim_mx4_linear_grad_workspace", "sim_mx4_linear_grad", "sim_moe_route_workspace", "sim_moe_route", "sim_moe_route_grad", "sim_moe_layer_workspace",
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
        L.sim_mx4_linear_workspace.argtypes = [i64, i64, i64]
        L.sim_mx4_linear_workspace.restype = sz
        L.sim_mx4_matmul.argtypes = [P, P, P, P, P, i64, i64, i64, P, i32, i64]
        L.sim_mx4_linear.argtypes = [P, P, i32, i64, P, P, i64, i64, i64, P, i32, i64, P, sz]
        L.sim_mx4_linear_grad_workspace.argtypes = [i64, i64, i64]
        L.sim_mx4_linear_grad_workspace.restype = sz
        L.sim_mx4_linear_grad.argtypes = [P, i32, P, i64, P, i64, P, i64, i64, i64, i64, P, i64, P, i64, P, sz]
        L.sim_moe_route_workspace.argtypes = [i64, i32, i32]
        L.sim_moe_route_workspace.restype = sz
        L.sim_moe_route.argtypes = [P, P, i32, i64, i32, i64, P, i64, i32, i32, P, P, P, P, P, sz]
        L.sim_moe_route_grad.argtypes = [P, P, i32, i64, i32, i64, P, i64, i32, i32, P, P, P]
        L.sim_moe_layer_workspace.argtypes = [i64, i64, i32, i32, i64]
        L.sim_moe_layer_workspace.restype = sz
        L.sim_moe_layer.argtypes = [P, P, i32, i64, i64, i64, P, i32, i32, i64, P, i64, i32, i32, P, P, P, P, i32,
                                    i64, P, i64, P, sz]
        for name in ("sim_mx4_quantize", "sim_mx4_dequantize", "sim_mx4_matmul", "sim_mx4_linear", "sim_mx4_linear_grad",
                     "sim_moe_route", "sim_moe_route_grad", "sim_moe_layer"):
            getattr(L, name).restype = C.c_int
        L.sim_ops_last_error.argtypes = []
        L.sim_ops_last_error.restype = C.c_char_p
        _lib = L
    return _lib


_raw_stream = torch._C._cuda_getCurrentRawStream   # what current_stream(i).cuda_stream is, without the object
_device_now = torch._C._cuda_getDevice


def _call(dev, fn, *args):
    """fn(current stream of GPU dev, *args) with that GPU current."""
    if dev == _device_now():
        st = fn(_raw_stream(dev), *args)
    else:
        with torch.cuda.device(dev):
            st = fn(_raw_stream(dev), *args)
    if st != SIM_OK:
        raise SimError(st, lib().sim_ops_last_error().decode())


def _need(ok, why):
    if not ok:
        raise SimError(SIM_ERR_INVALID_ARG, why)


def _rows(x, what):
    """(type, rows, columns, row stride, GPU) of a matrix whose rows are contiguous."""
    t, dev = _TYPE.get(x.dtype), x.get_device()
    if t is None or dev < 0 or x.dim() != 2:
        _need(x.dim() == 2, f"{what} must have two dimensions")
        _need(t is not None, f"{what} must be float32, float16 or bfloat16")
        _need(False, f"{what} must be on the GPU")
    rows, cols = x.shape
    stride, step = x.stride()
    if (step != 1 and cols > 1) or (stride < cols and rows > 1):
        _need(False, f"the rows of {what} must be contiguous and must not overlap")
    return t, rows, cols, stride if stride > cols else cols, dev


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


def _stored(q, what):
    """(rows, columns, GPU) of a 4-bit tensor whose arrays are as they must be."""
    codes, scales, shape = q
    K = shape[-1]
    rows = shape[0] if len(shape) == 2 else math.prod(shape[:-1])
    groups, dev = (K + 255) // 256, codes.get_device()
    if not (codes.shape == (rows, groups * 128) and scales.shape == (rows, groups * 8) and codes.dtype is torch.uint8
            and scales.dtype is torch.uint8 and codes.is_contiguous() and scales.is_contiguous() and dev >= 0
            and scales.get_device() == dev):
        _need(False, f"codes and scales of {what} must be contiguous uint8 [{rows}, {groups * 128}] and "
                     f"[{rows}, {groups * 8}] on one GPU")
    return rows, K, dev


def mx4_quantize(x, transpose=False) -> Mx4:
    """``x`` [..., K] in 4 bits, a scale for 32 elements along its last axis.
    With ``transpose`` (two dimensions) the result is that of ``x.t()``."""
    shape = tuple(x.shape)
    if len(shape) != 2:
        _need(len(shape) > 0 and not transpose, "x needs a dimension, and two to be transposed")
        x = x.reshape(math.prod(shape[:-1]), shape[-1])
    t, rows, cols, stride, dev = _rows(x, "x")
    R, K = (cols, rows) if transpose else (rows, cols)
    groups = (K + 255) // 256
    codes = x.new_empty((R, groups * 128), dtype=torch.uint8)
    scales = x.new_empty((R, groups * 8), dtype=torch.uint8)
    _call(dev, lib().sim_mx4_quantize, x.data_ptr(), t, rows, cols, stride, 1 if transpose else 0, codes.data_ptr(),
          scales.data_ptr())
    return Mx4(codes, scales, (R, K) if transpose else shape)


def mx4_dequantize(q: Mx4, dtype=torch.bfloat16):
    """The values that ``q`` stands for."""
    rows, K, dev = _stored(q, "q")
    t = _TYPE.get(dtype)
    _need(t is not None, "dtype must be float32, float16 or bfloat16")
    out = q.codes.new_empty(q.shape, dtype=dtype)
    _call(dev, lib().sim_mx4_dequantize, q.codes.data_ptr(), q.scales.data_ptr(), rows, K, out.data_ptr(), t, K)
    return out


def mx4_matmul(a, b: Mx4, dtype=torch.bfloat16, out=None):
    """``a @ b.T`` with both in 4 bits along their last axis, summed in 32
    bits.  ``a`` [M, K] is an ``Mx4``, or a plain tensor that is put into 4
    bits on the way; ``b`` [N, K]; the result is [M, N] of ``dtype`` (or of
    ``out``, which may have strided rows)."""
    _need(isinstance(b, Mx4) and len(b.shape) == 2, "b must be a 4-bit matrix")
    N, K, dev = _stored(b, "b")
    L = lib()
    plain = not isinstance(a, Mx4)
    if plain:
        at, M, Ka, stride, adev = _rows(a, "a")
    else:
        _need(len(a.shape) == 2, "a must be a matrix")
        M, Ka, adev = _stored(a, "a")
    _need(Ka == K and adev == dev, "a and b differ in their last axis or their GPU")
    if out is None:
        t = _TYPE.get(dtype)
        _need(t is not None, "dtype must be float32, float16 or bfloat16")
        out, ostride = b.codes.new_empty((M, N), dtype=dtype), N
    else:
        t, m, cols, ostride, odev = _rows(out, "out")
        _need(m == M and cols == N and odev == dev, "out must be [M, N] on the same GPU")
    if plain:
        n = L.sim_mx4_linear_workspace(M, N, K)
        ws = b.codes.new_empty(n) if n else None
        _call(dev, L.sim_mx4_linear, a.data_ptr(), at, stride, b.codes.data_ptr(), b.scales.data_ptr(), M, N, K, out.data_ptr(),
              t, ostride, ws.data_ptr() if n else None, n)
    else:
        _call(dev, L.sim_mx4_matmul, a.codes.data_ptr(), a.scales.data_ptr(), b.codes.data_ptr(), b.scales.data_ptr(), M, N, K,
              out.data_ptr(), t, ostride)
    return out


def mx4_linear_grad(dy, x, w, need=(True, True)):
    """Gradients ``(dx, dw)`` of ``y = x @ w.T`` computed in 4 bits, where
    rounding to 4 bits passes gradients through: ``dx = dy @ w`` and ``dw =
    dy.T @ x``, each operand quantised along the axis that is summed over.
    All of one type.  ``need``: which of the two to compute (None where not)."""
    (t, M, N, ys, dev), (tx, xm, K, xs, d1), (tw, wn, wk, ws, d2) = _rows(dy, "dy"), _rows(x, "x"), _rows(w, "w")
    _need(M == xm and N == wn and K == wk and dev == d1 == d2, "dy, x and w do not fit together")
    _need(t == tx == tw, "dy, x and w must have one type")
    dx = x.new_empty((M, K)) if need[0] else None
    dw = x.new_empty((N, K)) if need[1] else None
    L = lib()
    n = L.sim_mx4_linear_grad_workspace(M, N, K)
    space = x.new_empty(n, dtype=torch.uint8) if n else None
    _call(dev, L.sim_mx4_linear_grad, t, dy.data_ptr(), ys, x.data_ptr(), xs, w.data_ptr(), ws, M, N, K,
          dx.data_ptr() if need[0] else None, K, dw.data_ptr() if need[1] else None, K, space.data_ptr() if n else None, n)
    return dx, dw


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return mx4_matmul(x, mx4_quantize(w), dtype=x.dtype)

    @staticmethod
    def backward(ctx, dy):
        return mx4_linear_grad(dy.contiguous(), *ctx.saved_tensors, need=ctx.needs_input_grad)


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
    """(pointer, type, T, E, row stride, mask pointer, mask stride, k), GPU"""
    t, T, E, stride, dev = _rows(logits, "logits")
    _need(1 <= k <= E and k <= MAX_TOPK, "k out of range")
    mptr, mstride = None, 0
    if mask is not None:
        _need(mask.dtype in (torch.bool, torch.uint8) and mask.get_device() == dev, "mask must be bool or uint8 on the same GPU")
        _need(tuple(mask.shape) in ((E,), (T, E)), "mask must be [E] or [T, E]")
        _need(E == 1 or mask.stride(-1) == 1, "mask must have contiguous rows")
        if mask.dim() == 2:
            mstride = mask.stride(0)  # 0 where one row is expanded over the tokens
            _need(T <= 1 or mstride == 0 or mstride >= E, "the rows of mask must not overlap")
        mptr = mask.data_ptr()
    return (logits.data_ptr(), t, T, E, stride, mptr, mstride, k), dev


def moe_route(logits, k, mask=None, renormalize=True) -> Routes:
    """The k experts of each token with the highest logits [T, E], their
    softmax weights, and the experts' lists of slots.  ``mask`` ([E] or [T,
    E], true = allowed) takes experts out; ``renormalize`` divides a token's
    weights by their sum."""
    args, dev = _route_args(logits, k, mask)
    T, E = args[2], args[3]
    slots = T * k
    experts = logits.new_empty((T, k), dtype=torch.int32)
    weights = logits.new_empty((T, k), dtype=torch.float32)
    offsets = logits.new_empty(E + 1, dtype=torch.int32)
    order = logits.new_empty(slots, dtype=torch.int32)
    L = lib()
    n = L.sim_moe_route_workspace(T, E, k)
    ws = logits.new_empty(n, dtype=torch.uint8) if n else None
    _call(dev, L.sim_moe_route, *args, 1 if renormalize else 0, experts.data_ptr(), weights.data_ptr(), offsets.data_ptr(),
          order.data_ptr() if slots else None, ws.data_ptr() if n else None, n)
    return Routes(experts, weights, offsets, order)


def moe_route_grad(logits, experts, d_weights, mask=None, renormalize=True):
    """Gradient of ``moe_route``'s weights with respect to the logits, from
    the gradient [T, k] of the weights."""
    _need(experts.dim() == 2, "experts must be [T, k]")
    T, k = experts.shape
    args, dev = _route_args(logits, k, mask)
    _need(args[2] == T and d_weights.shape == experts.shape, "experts and d_weights must be [T, k]")
    _need(experts.dtype is torch.int32 and d_weights.dtype is torch.float32, "experts must be int32, d_weights float32")
    _need(experts.is_contiguous() and d_weights.is_contiguous(), "experts and d_weights must be contiguous")
    _need(experts.get_device() == dev and d_weights.get_device() == dev, "tensors are on different GPUs")
    dz = logits.new_empty((T, args[3]))
    _call(dev, lib().sim_moe_route_grad, *args, 1 if renormalize else 0, experts.data_ptr(), d_weights.data_ptr(),
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
    t, T, D, xstride, dev = _rows(x, "x")
    _need(t != 0, "x must be float16 or bfloat16")
    (lptr, lt, lT, E, lstride, mptr, mstride, k), ldev = _route_args(logits, k, mask)
    _need(lT == T and ldev == dev, "x and logits differ in their tokens or their GPU")
    mx4 = isinstance(w13, Mx4)
    s13, s2 = tuple(w13.shape), tuple(w2.shape)
    _need(mx4 == isinstance(w2, Mx4) and len(s2) == 3, "w13 must be [E, 2F, D], w2 [E, D, F], of one kind")
    F = s2[2]
    _need(s13 == (E, 2 * F, D) and s2 == (E, D, F), "w13 must be [E, 2F, D], w2 [E, D, F]")
    if mx4:
        same = _stored(w13, "w13")[2] == _stored(w2, "w2")[2] == dev
        wargs = (w13.codes.data_ptr(), w13.scales.data_ptr(), w2.codes.data_ptr(), w2.scales.data_ptr(), _MX4)
    else:
        _need(w13.dtype is x.dtype and w2.dtype is x.dtype, "the weights must have the type of x or be in 4 bits")
        _need(w13.is_contiguous() and w2.is_contiguous(), "the weights must be contiguous")
        same = w13.get_device() == w2.get_device() == dev
        wargs = (w13.data_ptr(), None, w2.data_ptr(), None, t)
    _need(same, "tensors are on different GPUs")
    if out is None:
        out, ostride = x.new_empty((T, D)), D
    else:
        ot, m, cols, ostride, odev = _rows(out, "out")
        _need(ot == t and m == T and cols == D and odev == dev, "out must be like x")
    L = lib()
    n = L.sim_moe_layer_workspace(T, D, E, k, F)
    ws = x.new_empty(n, dtype=torch.uint8) if n else None
    _call(dev, L.sim_moe_layer, x.data_ptr(), t, T, D, xstride, lptr, lt, E, lstride, mptr, mstride, k,
          1 if renormalize else 0, *wargs, F, out.data_ptr(), ostride, ws.data_ptr() if n else None, n)
    return out
