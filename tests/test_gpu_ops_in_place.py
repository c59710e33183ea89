"""Results written where the call's input stands, or beside it in one buffer."""
from __future__ import annotations

import pytest

from tests.test_gpu_ops import layer_case, ops, rand  # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# one launch that puts a into 4 bits itself (at most 16384 elements), one after another, and tiles
@pytest.mark.parametrize("M,K", [(1, 64), (4, 300), (4, 4096), (16, 1024), (31, 513), (20, 4096), (70, 300), (300, 513)])
@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
def test_linear_in_place(ops, kind, M, K):  # noqa: F811
    x, _ = rand(80, (M, K), kind)
    w = ops.mx4_quantize(rand(81, (K, K), "bf16", scale=K ** -0.5)[0])
    want = ops.mx4_matmul(x, w, dtype=x.dtype)
    got = x.clone()
    assert ops.mx4_matmul(got, w, out=got) is got
    assert torch.equal(got, want)


@pytest.mark.parametrize("M", [3, 40])
def test_linear_beside_its_input_and_over_a_part_of_it(ops, M):  # noqa: F811
    x, _ = rand(82, (M, 256), "bf16")
    w = ops.mx4_quantize(rand(83, (96, 256), "bf16", scale=1 / 16)[0])
    want = ops.mx4_matmul(x, w)
    both = torch.empty(M, 400, dtype=x.dtype, device="cuda")
    both[:, :256] = x
    ops.mx4_matmul(both[:, :256], w, out=both[:, 256:352])
    assert torch.equal(both[:, 256:352], want) and torch.equal(both[:, :256], x)
    ops.mx4_matmul(both[:, :256], w, out=both[:, 200:296])
    assert torch.equal(both[:, 200:296], want) and torch.equal(both[:, :200], x[:, :200])


@pytest.mark.parametrize("T", [1, 5, 16, 40, 200])
@pytest.mark.parametrize("weights", ["same", "mx4"])
def test_layer_in_place(ops, weights, T):  # noqa: F811
    (x, z, w13, w2), _ = layer_case(ops, 84, T, 6, 320, 96, "bf16", weights)
    want = ops.moe_layer(x, z, w13, w2, 2)
    assert ops.moe_layer(x, z, w13, w2, 2, out=x) is x
    assert torch.equal(x, want)
