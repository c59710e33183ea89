"""Operators where offsets pass 31 and 32 bits: rows far apart, large results,
the last of many experts.  Bounds are those of ``ops_reference``."""
from __future__ import annotations

import numpy as np
import pytest

from tests import ops_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
FAR = (1 << 31) + 40  # elements


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    yield o
    torch.cuda.empty_cache()


def rand(seed, shape, scale=1.0):
    v = torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * scale).to(torch.bfloat16)
    return v.cuda(), v.double().numpy()


def far_rows(x):
    """The same rows, FAR elements apart."""
    wide = torch.empty((len(x) - 1) * FAR + x.shape[1], dtype=x.dtype, device="cuda")
    out = wide.as_strided(x.shape, (FAR, 1))
    out.copy_(x)
    return out


def check(got, want, bound):
    off = np.abs(got.double().cpu().numpy() - want)
    assert off.shape == want.shape and (off <= bound).all()


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_rows_far_apart(ops, transpose):
    x, v = rand(1, (3, 300))
    q = ops.mx4_quantize(far_rows(x), transpose=transpose)
    codes, scales = ref.mx4_stored(v.T if transpose else v)
    assert np.array_equal(q.codes.cpu().numpy(), codes) and np.array_equal(q.scales.cpu().numpy(), scales)


def test_linear_and_its_result_of_rows_far_apart(ops):
    (x, vx), (w, vw) = rand(2, (3, 300)), rand(3, (70, 300))
    out = far_rows(torch.zeros(3, 70, dtype=x.dtype, device="cuda"))
    ops.mx4_matmul(far_rows(x), ops.mx4_quantize(w), out=out)
    check(out, *ref.product(ref.mx4_values(vx), ref.mx4_values(vw), "bf16"))


def test_router_rows_far_apart(ops):
    z, v = rand(4, (3, 20))
    far = far_rows(z)
    r = ops.moe_route(far, 4)
    experts, weights, offsets, order, rel = ref.route(v, 4, None, True)
    assert np.array_equal(r.experts.cpu().numpy(), experts) and np.array_equal(r.order.cpu().numpy(), order)
    check(r.weights, weights, rel * weights)
    dw = torch.ones(3, 4, device="cuda") * torch.arange(4, device="cuda")
    assert torch.equal(ops.moe_route_grad(far, r.experts, dw), ops.moe_route_grad(z, r.experts, dw))


def test_dequantize_many_rows(ops):
    K, R = 257, (1 << 23) + 70  # codes and results past 2^31 bytes and elements
    v = np.random.default_rng(5).standard_normal((3, K))
    codes, scales = ref.mx4_stored(v)
    q = ops.Mx4(torch.zeros(R, codes.shape[1], dtype=torch.uint8, device="cuda"),
                torch.zeros(R, scales.shape[1], dtype=torch.uint8, device="cuda"), (R, K))
    q.codes[-3:], q.scales[-3:] = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    out = ops.mx4_dequantize(q, torch.bfloat16)
    assert np.array_equal(out[-3:].double().cpu().numpy(), ref.mx4_values(v))
    assert not out[:3].any() and not out[-6:-3].any()


def test_product_with_a_large_result(ops):
    n, K = 66000, 32
    (a, va), (b, vb) = rand(6, (n, K)), rand(7, (n, K))
    out = ops.mx4_matmul(ops.mx4_quantize(a), ops.mx4_quantize(b))
    rows = [0, 1, 32768, 65535, 65999]
    check(torch.stack([out[i] for i in rows]), *ref.product(ref.mx4_values(va[rows]), ref.mx4_values(vb), "bf16"))


@pytest.mark.parametrize("weights", ["same", "mx4"])
@pytest.mark.parametrize("T", [2, 17])
def test_layer_last_of_many_experts(ops, weights, T):
    E, D, F = 256, 4096, 2176
    x, vx = rand(8, (T, D))
    (a, va), (b, vb) = rand(9, (2 * F, D), D ** -0.5), rand(10, (D, F), F ** -0.5)

    def at_the_end(last):
        all_ = torch.zeros((E,) + last.shape, dtype=last.dtype, device="cuda")
        all_[-1] = last
        return all_

    if weights == "mx4":
        w13, w2 = (ops.Mx4(at_the_end(q.codes).flatten(0, 1), at_the_end(q.scales).flatten(0, 1), (E,) + q.shape)
                   for q in (ops.mx4_quantize(a), ops.mx4_quantize(b)))
        va, vb = ref.mx4_values(va), ref.mx4_values(vb)
    else:
        w13, w2 = at_the_end(a), at_the_end(b)
    only = torch.zeros(E, dtype=torch.bool, device="cuda")
    only[-1] = True
    y = ops.moe_layer(x, torch.zeros(T, E, device="cuda"), w13, w2, 1, mask=only)
    some = [0, T - 1]
    check(y[some], *ref.layer(vx[some], np.zeros((2, 1)), va[None], vb[None], 1, None, True, "bf16"))
