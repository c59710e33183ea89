"""The router with scores where there are more tokens than one workgroup takes a wave each for: large k, many experts, groups
of every kind; choices and lists exactly."""
from __future__ import annotations

import numpy as np
import pytest

from tests import route_reference as ref
from tests.test_gpu_route_scores import TYPES, check, logits, masks

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


def run(ops, T, E, groups, top_groups, best, k, kind, score, biased, how="", renorm=True, scale=2.5):
    z, v = logits(T + E + k, T, E, kind, pad=3)
    mask, m = masks(k, T, E, how)
    bias = np.random.default_rng(k).standard_normal(E).astype(np.float32) * 0.1 if biased else None
    r = ops.moe_route(z, k, mask, renorm, score=score, bias=None if bias is None else torch.from_numpy(bias).cuda(), groups=groups,
                      top_groups=top_groups, group_best=best, scale=scale)
    check(r, ref.route(v, k, m, renorm, score, bias, groups, top_groups, best, scale))


@pytest.mark.parametrize("biased", [True, False])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("k", [14, 15, 16, 17, 31, 32])
@pytest.mark.parametrize("T,E", [(17, 32), (17, 1024), (64, 60), (70, 64), (70, 256), (70, 700)])
def test_large_k(ops, T, E, k, score, biased):
    run(ops, T, E, 1, 1, 1, k, "fp32", score, biased)
    run(ops, T, E, 1, 1, 1, k, "bf16", score, biased, "token", False)
    if E % 4 == 0 and E // 2 >= k:
        run(ops, T, E, 4, 2, 2, k, "fp32", score, biased)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("biased", [True, False])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T", [17, 70])
@pytest.mark.parametrize("shape", [(8, 4, 2, 2, 3), (16, 16, 5, 2, 5), (30, 30, 4, 2, 4), (36, 2, 1, 2, 18), (60, 5, 2, 2, 4), (64, 64, 10, 2, 10), (96, 3, 2, 2, 7),
                                   (160, 8, 3, 1, 6), (256, 16, 5, 1, 9), (512, 64, 9, 2, 17), (640, 64, 6, 1, 9), (700, 7, 3, 2, 17), (1024, 16, 3, 2, 32),
                                   (1024, 64, 10, 1, 32)])
def test_shapes(ops, kind, score, biased, T, shape):
    E, groups, top_groups, best, k = shape
    run(ops, T, E, groups, top_groups, best, k, kind, score, biased, "token" if T == 70 else "", T == 17)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("k", [15, 32])
def test_many_tokens_with_many_choices(ops, score, k):
    run(ops, 4200, 64, 4, 3, 2, k, "fp32", score, True, "token")


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("k", [14, 16, 31, 32])
def test_biases_a_rounding_apart(ops, score, k):
    # the choice depends on the last place of a score and its sum with the bias, down to the last one chosen and the next
    g = np.random.default_rng(k)
    T, E = 40, 64
    b = (0.25 + g.integers(0, 12, E) * 2.0 ** -25).astype(np.float32)
    v = np.full((T, E), 0.3, np.float32)
    v[1::2] = np.nextafter(np.float32(1.25), np.float32(2)) + g.integers(0, 6, (T // 2, E)).astype(np.float32) * np.float32(2.0 ** -23)
    r = ops.moe_route(torch.from_numpy(v).cuda(), k, score=score, bias=torch.from_numpy(b).cuda())
    check(r, ref.route(v.astype(np.float64), k, None, True, score, b))
