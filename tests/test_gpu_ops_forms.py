"""Each form of the operators' kernels, at sizes that run it (which size runs
which form is checked on the CPU, ``test_ops_forms``): products by whole
numbers, whose every partial sum is exact, so that each element, scale and
stage shows; the few tokens' layer with its inputs in LDS and past it."""
from __future__ import annotations

import numpy as np
import pytest

from tests import ops_reference as ref
from tests.test_gpu_ops import TYPES, check, layer_case, ops  # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# M, N, K: remainders of the tile in M and N, of 32 and 256 in K; two stages and many, an odd number of groups and an even one
TILE_K = [31, 256, 300, 513, 1025, 2304, 2311]
PRODUCTS = {
    "skinny_small": [(1, 333, 2311), (16, 95, 4096), (17, 70, 5000), (32, 161, 2311)],
    "skinny_large": [(32, 333, 4096), (17, 70, 6001), (16, 95, 9000), (16, 40, 16384), (1, 33, 200001), (31, 64, 8191)],
    "64x64": [(65, 200, k) for k in TILE_K] + [(333, 1001, 2311), (1, 3, (1 << 20) + 100), (32, 70, 16384)],
    "64x128": [(333, 5001, k) for k in TILE_K],
    "128x128": [(900, 3300, k) for k in TILE_K],
    "256x256": [(2051, 6301, k) for k in (31, 300, 513, 2304, 2311)],
    "simple": [(2, 3, (1 << 23) + 300), (1, 9, 1 << 23)],
}
CASES = [(form, *mnk) for form, cases in PRODUCTS.items() for mnk in cases]


def whole(seed, R, K):
    """R x K whole numbers that 4 bits hold exactly, in blocks of two sizes; products of K of them stay below 2^24."""
    rng = np.random.default_rng(seed)
    if K >= 1 << 23:
        return rng.integers(-1, 2, (R, K), np.int8).astype(np.float32)
    if K >= 1 << 17:
        return rng.integers(-2, 3, (R, K), np.int8).astype(np.float32)
    v = rng.choice(np.array([-6, -4, -3, -2, -1, 0, 1, 2, 3, 4, 6], np.float32), (R, K))
    return v * np.repeat(rng.integers(1, 3, (R, -(-K // 32))), 32, axis=1)[:, :K].astype(np.float32)


def exact(a, b):
    most = float(np.abs(a).max()) * float(np.abs(b).max()) * a.shape[1]
    assert most < 2 ** 24
    return a.astype(np.float64) @ b.astype(np.float64).T


@pytest.mark.parametrize("form,M,N,K", CASES)
def test_product(ops, form, M, N, K):  # noqa: F811
    a, b = whole(1, M, K), whole(2, N, K)
    qa, qb = (ops.mx4_quantize(torch.from_numpy(v).cuda()) for v in (a, b))
    assert torch.equal(ops.mx4_dequantize(qa, torch.float32), torch.from_numpy(a).cuda())
    want = torch.from_numpy(exact(a, b)).cuda()
    for kind in TYPES.values():
        wide = torch.full((M, N + 3), 7.0, dtype=kind, device="cuda")
        ops.mx4_matmul(qa, qb, out=wide[:, :N])
        assert torch.equal(wide[:, :N], want.to(kind)), kind
        assert (wide[:, N:] == 7.0).all()
    if form in ("skinny_small", "64x64"):
        assert torch.equal(ops.mx4_matmul(torch.from_numpy(a).cuda(), qb, dtype=torch.float32), want.float())


# at most 16384 elements: put into 4 bits by every workgroup
IN_ONE = [(1, 33, 16384), (1, 50, 15999), (2, 70, 8192), (16, 95, 1024), (17, 40, 900), (31, 50, 528), (32, 70, 512)]


@pytest.mark.parametrize("M,N,K", IN_ONE)
@pytest.mark.parametrize("kind", TYPES)
def test_linear_in_one_launch(ops, kind, M, N, K):  # noqa: F811
    a, b = whole(3, M, K), whole(4, N, K)
    x = torch.full((M, K + 5), float("nan"), dtype=TYPES[kind], device="cuda")
    x[:, :K] = torch.from_numpy(a).cuda()
    got = ops.mx4_matmul(x[:, :K], ops.mx4_quantize(torch.from_numpy(b).cuda()), dtype=torch.float32)
    assert torch.equal(got, torch.from_numpy(exact(a, b)).cuda().float())


@pytest.mark.parametrize("form", ["64x128", "128x128", "256x256"])
def test_nan_stays_in_its_row_and_column(ops, form):  # noqa: F811
    M, N, K = PRODUCTS[form][-1]
    a, b = whole(5, M, K), whole(6, N, K)
    a[M - 2, K - 1] = float("inf")
    b[37, 290] = float("nan")
    got = ops.mx4_matmul(*(ops.mx4_quantize(torch.from_numpy(v).cuda()) for v in (a, b)), dtype=torch.float32)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[M - 2], bad[:, 37] = True, True
    assert torch.equal(torch.isnan(got), bad)


# ------------------------------------------------------------------ the layer for few tokens

# T, E, k, D, F: all tokens go to the first k - 1 experts, the last choice is spread over the others
PAST_LDS = [(16, 3, 2, 2053, 70), (16, 2, 2, 1024, 96), (12, 5, 3, 1216, 41), (9, 4, 2, 4096, 33), (16, 16, 4, 1029, 900)]
COLS = {"same": 64, "mx4": 128}  # columns of a step


def spread(T, E, k, turned):
    """Logits with that choice; turned: the common experts are the last ones, so that other workgroups meet them."""
    z = np.random.default_rng(7).standard_normal((T, E)) * 0.1
    z[:, :k - 1] += 4.0
    z[np.arange(T), k - 1 + np.arange(T) % (E - k + 1)] += 2.0
    return (z[:, ::-1] if turned else z).copy()


def tokens_of_experts(z, k):
    top = np.argsort(-z, axis=1, kind="stable")[:, :k]
    return np.bincount(top.reshape(-1), minlength=z.shape[1])


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("weights", ["same", "mx4"])
@pytest.mark.parametrize("case", PAST_LDS)
@pytest.mark.parametrize("turned", [False, True])
def test_layer_inputs_past_lds(ops, kind, weights, case, turned):  # noqa: F811
    T, E, k, D, F = case
    (x, _, w13, w2), (vx, _, v13, v2) = layer_case(ops, 90, T, E, D, F, kind, weights, pad=3)
    z = torch.from_numpy(spread(T, E, k, turned)).float()
    got = ops.moe_layer(x, z.cuda(), w13, w2, k)
    check(got, *ref.layer(vx, z.double().numpy(), v13, v2, k, None, True, kind))
