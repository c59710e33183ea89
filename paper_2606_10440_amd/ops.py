"""Operators of an expert-parallel step on the GPU, next to the traffic that
``sim`` simulates: 4-bit microscaled tensors (what travels, and the products of
linear layers), the router with the experts' token lists (who gets it), and
the experts' layer for few tokens (what is computed there).

Functions marshal torch tensors for the C ABI of ``include/simgpu_ops.h``
(there the layouts, formulas and limits are stated), by way of
``csrc/ops_torch.cpp``.  Work is enqueued on the current stream of the
tensors' device; results and workspaces come from torch's allocator, so a call
may be captured into a graph.  Every step runs in the library's HIP kernels;
there is no host or torch fallback.  Refused arguments raise ``SimError``
before anything is enqueued.

Results carry no gradients, whatever the arguments require, but those of
``mx4_linear`` and ``moe_route_train``.  ``out`` must not require one.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch
from torch.autograd.function import once_differentiable

from . import sim
from .sim import SimError

EXPORTS = ("sim_mx4_code_pitch", "sim_mx4_scale_pitch", "sim_mx4_quantize", "sim_mx4_dequantize",
           "sim_mx4_matmul", "sim_mx4_linear_workspace", "sim_mx4_linear",
           "sim_mx4_linear_grad_workspace", "sim_mx4_linear_grad", "sim_moe_route_workspace", "sim_moe_route",
           "sim_moe_route_grad", "sim_moe_layer_workspace", "sim_moe_layer", "sim_ops_last_error")

MAX_EXPERTS, MAX_TOPK, MAX_LAYER_TOKENS = 1024, 32, 1024

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


_torch = None


def _c():
    """The binding to torch tensors, on the functions of libsimgpu.so."""
    global _torch
    if _torch is None:
        L = lib()
        try:
            from . import _ops_torch
        except ImportError as e:
            raise RuntimeError("_ops_torch.so is missing or does not load: build it with paper_2606_10440_amd/build.py") from e
        _ops_torch.setup(SimError, Mx4, Routes, {name: C.cast(getattr(L, name), C.c_void_p).value for name in EXPORTS})
        _torch = _ops_torch
    return _torch


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


def mx4_quantize(x, transpose=False) -> Mx4:
    """``x`` [..., K] in 4 bits, a scale for 32 elements along its last axis.
    With ``transpose`` (two dimensions) the result is that of ``x.t()``."""
    return _c().quantize(x, transpose)


def mx4_dequantize(q: Mx4, dtype=torch.bfloat16):
    """The values that ``q`` stands for."""
    return _c().dequantize(q, dtype)


def mx4_matmul(a, b: Mx4, dtype=torch.bfloat16, out=None):
    """``a @ b.T`` with both in 4 bits along their last axis, summed in 32
    bits.  ``a`` [M, K] is an ``Mx4``, or a plain tensor that is put into 4
    bits on the way; ``b`` [N, K]; the result is [M, N] of ``dtype`` (or of
    ``out``, which may have strided rows, and may be a plain ``a``)."""
    return _c().matmul(a, b, dtype, out)


def mx4_linear_grad(dy, x, w, need=(True, True)):
    """Gradients ``(dx, dw)`` of ``y = x @ w.T`` computed in 4 bits, where
    rounding to 4 bits passes gradients through: ``dx = dy @ w`` and ``dw =
    dy.T @ x``, each operand quantised along the axis that is summed over.
    All of one type.  ``need``: which of the two to compute (None where not)."""
    return _c().linear_grad(dy, x, w, *need)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        if x.dtype != w.dtype:  # the gradient would be refused, a whole forward pass later
            raise SimError(sim.SIM_ERR_INVALID_ARG, "mx4_linear: x and w must have one type")
        ctx.save_for_backward(x, w)
        return mx4_matmul(x, mx4_quantize(w), dtype=x.dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        return mx4_linear_grad(dy.contiguous(), *ctx.saved_tensors, need=ctx.needs_input_grad)


def mx4_linear(x, w):
    """``x @ w.T`` with both put into 4 bits, for training: x [M, K] and w
    [N, K], of one type, get the gradients of ``mx4_linear_grad`` (which have
    none themselves)."""
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


def moe_route(logits, k, mask=None, renormalize=True) -> Routes:
    """The k experts of each token with the highest logits [T, E], their
    softmax weights, and the experts' lists of slots.  ``mask`` ([E] or [T,
    E], true = allowed) takes experts out; ``renormalize`` divides a token's
    weights by their sum."""
    return _c().route(logits, k, mask, renormalize)


def moe_route_grad(logits, experts, d_weights, mask=None, renormalize=True):
    """Gradient of ``moe_route``'s weights with respect to the logits, from
    the gradient [T, k] of the weights."""
    return _c().route_grad(logits, experts, d_weights, mask, renormalize)


class _RouteWeights(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, mask, renormalize):
        r = moe_route(logits, k, mask, renormalize)
        ctx.save_for_backward(logits, r.experts, mask)
        ctx.renormalize = renormalize
        ctx.mark_non_differentiable(r.experts, r.offsets, r.order)
        return r.experts, r.weights, r.offsets, r.order

    @staticmethod
    @once_differentiable
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
    is float16 or bfloat16; the weights have its type, or are ``Mx4``; ``out``
    may be x.  For inference: the result carries no gradients."""
    return _c().layer(x, logits, w13, w2, k, mask, renormalize, out)
