"""Operators without a GPU: the library exports what its header declares, and
refused arguments come back as errors before any device work."""
from __future__ import annotations

import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2606_10440_amd import ops, sim
    if not os.path.exists(sim.LIB_PATH):
        from paper_2606_10440_amd import build
        build.build()
    return ops.lib()


def test_exports_match_header(lib):
    from paper_2606_10440_amd import ops
    hdr = open(os.path.join(ROOT, "include", "simgpu_ops.h")).read()
    declared = set(re.findall(r"^\s*(?:sim_status|const char \*|size_t|int64_t)\s*(sim_\w+)\s*\(", hdr, re.M))
    assert declared == set(ops.EXPORTS)
    for name in declared:
        assert hasattr(lib, name), name


def test_pitches(lib):
    for K, g in [(0, 0), (1, 1), (256, 1), (257, 2), (4096, 16)]:
        assert lib.sim_mx4_code_pitch(K) == g * 128 and lib.sim_mx4_scale_pitch(K) == g * 8


P = 1 << 20          # an aligned address that is never read: the calls below are refused
INVALID, SIZE = 1, 4


def run(lib, name, args, **change):
    names, values = zip(*args)
    values = [change.get(n, v) for n, v in args]
    assert set(change) <= set(names)
    st = getattr(lib, name)(None, *values)
    if st:
        assert lib.sim_ops_last_error().decode().startswith(name)
    return st


QUANT = [("x", P), ("type", 2), ("rows", 4), ("cols", 64), ("stride", 64), ("transpose", 0), ("codes", P), ("scales", P)]


@pytest.mark.parametrize("change,want", [
    (dict(x=None), INVALID), (dict(type=3), INVALID), (dict(type=-1), INVALID), (dict(rows=-1), INVALID),
    (dict(cols=-5), INVALID), (dict(stride=63), INVALID), (dict(transpose=2), INVALID), (dict(codes=None), INVALID),
    (dict(scales=None), INVALID), (dict(x=P + 1), INVALID), (dict(codes=P + 8), INVALID), (dict(scales=P + 4), INVALID),
    (dict(rows=1 << 40), SIZE), (dict(rows=1 << 30, cols=1 << 30, stride=1 << 30), SIZE), (dict(rows=0), 0), (dict(cols=0), 0)])
def test_quantize_refusals(lib, change, want):
    assert run(lib, "sim_mx4_quantize", QUANT, **change) == want


DEQUANT = [("codes", P), ("scales", P), ("rows", 4), ("cols", 64), ("out", P), ("type", 0), ("stride", 64)]


@pytest.mark.parametrize("change,want", [
    (dict(codes=None), INVALID), (dict(out=None), INVALID), (dict(type=3), INVALID), (dict(rows=-1), INVALID),
    (dict(stride=10), INVALID), (dict(out=P + 2), INVALID), (dict(codes=P + 1), INVALID), (dict(rows=0), 0)])
def test_dequantize_refusals(lib, change, want):
    assert run(lib, "sim_mx4_dequantize", DEQUANT, **change) == want


MATMUL = [("ac", P), ("as", P), ("bc", P), ("bs", P), ("M", 4), ("N", 8), ("K", 64), ("out", P), ("type", 2), ("stride", 8)]
# so many rows that they are put into 4 bits in a workspace
LINEAR = [("x", P), ("x_type", 2), ("x_stride", 64), ("wc", P), ("ws_", P), ("M", 40), ("N", 8), ("K", 64), ("out", P),
          ("type", 2), ("stride", 8), ("ws", P), ("ws_bytes", 1 << 30)]


@pytest.mark.parametrize("change,want", [
    (dict(ac=None), INVALID), (dict(bs=None), INVALID), (dict(out=None), INVALID), (dict(type=3), INVALID),
    (dict(M=-1), INVALID), (dict(K=-1), INVALID), (dict(stride=7), INVALID), (dict(bc=P + 8), INVALID), (dict(out=P + 1), INVALID),
    (dict(M=1 << 30, N=1 << 30, stride=1 << 30), SIZE), (dict(M=0), 0), (dict(N=0), 0)])
def test_product_refusals(lib, change, want):
    assert run(lib, "sim_mx4_matmul", MATMUL, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(x=None), INVALID), (dict(wc=None), INVALID), (dict(x_type=3), INVALID), (dict(x_stride=63), INVALID),
    (dict(stride=7), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=4), INVALID), (dict(ws=P + 4), INVALID),
    (dict(x=P + 1), INVALID), (dict(M=0), 0)])
def test_linear_refusals(lib, change, want):
    assert run(lib, "sim_mx4_linear", LINEAR, **change) == want


LGRAD = [("type", 2), ("dy", P), ("dy_stride", 8), ("x", P), ("x_stride", 64), ("w", P), ("w_stride", 64), ("M", 4), ("N", 8),
         ("K", 64), ("dx", P), ("dx_stride", 64), ("dw", P), ("dw_stride", 64), ("ws", P), ("ws_bytes", 1 << 30)]


@pytest.mark.parametrize("change,want", [
    (dict(type=3), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(M=-1), INVALID),
    (dict(dy_stride=7), INVALID), (dict(x_stride=63), INVALID), (dict(w_stride=63), INVALID), (dict(dx_stride=63), INVALID),
    (dict(dw_stride=63), INVALID), (dict(dx=P + 1), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=64), INVALID),
    (dict(N=1 << 31, dy_stride=1 << 31), SIZE), (dict(dx=None, dw=None), 0), (dict(K=0), 0)])
def test_linear_gradient_refusals(lib, change, want):
    assert run(lib, "sim_mx4_linear_grad", LGRAD, **change) == want


ROUTE = [("logits", P), ("type", 0), ("T", 100), ("E", 16), ("stride", 16), ("mask", None), ("mask_stride", 0), ("k", 2),
         ("renorm", 1), ("experts", P), ("weights", P), ("offsets", P), ("order", P), ("ws", P), ("ws_bytes", 1 << 20)]
ROUTE_BAD = [(dict(logits=None), INVALID), (dict(type=3), INVALID), (dict(T=-1), INVALID), (dict(E=0), INVALID),
             (dict(E=1025, stride=2000), INVALID), (dict(k=0), INVALID), (dict(k=17), INVALID), (dict(E=64, stride=64, k=33), INVALID),
             (dict(stride=15), INVALID), (dict(mask=P, mask_stride=15), INVALID), (dict(logits=P + 2), INVALID),
             (dict(T=1 << 30), SIZE)]


@pytest.mark.parametrize("change,want", ROUTE_BAD + [
    (dict(experts=None), INVALID), (dict(weights=None), INVALID), (dict(order=None), INVALID), (dict(offsets=None), INVALID),
    (dict(ws=None), INVALID), (dict(ws_bytes=0), INVALID)])
def test_route_refusals(lib, change, want):
    assert run(lib, "sim_moe_route", ROUTE, **change) == want


GRAD = ROUTE[:9] + [("experts", P), ("dw", P), ("dz", P)]


@pytest.mark.parametrize("change,want", ROUTE_BAD + [
    (dict(experts=None), INVALID), (dict(dw=None), INVALID), (dict(dz=None), INVALID), (dict(dz=P + 2), INVALID), (dict(T=0), 0)])
def test_route_gradient_refusals(lib, change, want):
    assert run(lib, "sim_moe_route_grad", GRAD, **change) == want


LAYER = [("x", P), ("type", 2), ("T", 4), ("D", 64), ("x_stride", 64), ("logits", P), ("logit_type", 0), ("E", 16),
         ("stride", 16), ("mask", None), ("mask_stride", 0), ("k", 2), ("renorm", 1), ("w13", P), ("s13", None), ("w2", P),
         ("s2", None), ("weight_type", 2), ("F", 32), ("y", P), ("y_stride", 64), ("ws", P), ("ws_bytes", 1 << 30)]


@pytest.mark.parametrize("change,want", [
    (dict(x=None), INVALID), (dict(type=0, weight_type=0), INVALID), (dict(weight_type=1), INVALID), (dict(weight_type=3), INVALID),
    (dict(s13=P), INVALID), (dict(w2=None), INVALID), (dict(T=1025), SIZE), (dict(D=1 << 20), SIZE), (dict(F=-1), INVALID),
    (dict(x_stride=63), INVALID), (dict(y_stride=63), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=100), INVALID),
    (dict(k=0), INVALID), (dict(E=2000, stride=2000), INVALID), (dict(w13=P + 1), INVALID), (dict(T=0), 0)])
def test_layer_refusals(lib, change, want):
    assert run(lib, "sim_moe_layer", LAYER, **change) == want


def test_workspace_queries_of_bad_sizes(lib):
    assert lib.sim_moe_route_workspace(-1, 16, 2) == 0 and lib.sim_moe_layer_workspace(-1, 64, 16, 2, 32) == 0
    assert lib.sim_moe_layer_workspace(2000, 64, 16, 2, 32) == 0 and lib.sim_mx4_linear_workspace(-1, 4, 4) == 0
    assert lib.sim_moe_layer_workspace(4, 64, 16, 2, 32) > 0


def test_binding_refuses_host_tensors(lib):
    torch = pytest.importorskip("torch")
    from paper_2606_10440_amd import SimError, ops
    x = torch.zeros(4, 64)
    for call in (lambda: ops.mx4_quantize(x), lambda: ops.mx4_quantize(torch.zeros(2, 3, 4), transpose=True),
                 lambda: ops.moe_route(x, 0), lambda: ops.moe_route(x, 65), lambda: ops.moe_route(x, 2),
                 lambda: ops.moe_layer(x, x, x, x, 2)):
        with pytest.raises(SimError):
            call()


@pytest.mark.parametrize("x,w", [("bfloat16", "float32"), ("float32", "float16")])
def test_linear_layer_refuses_types_that_its_gradient_refuses(x, w):
    import torch
    from paper_2606_10440_amd import ops
    from paper_2606_10440_amd.sim import SimError
    with pytest.raises(SimError, match="one type"):
        ops.mx4_linear(torch.zeros(2, 32, dtype=getattr(torch, x), requires_grad=True), torch.zeros(4, 32, dtype=getattr(torch, w)))
