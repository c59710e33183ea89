"""Calls on the paged cache that are refused: none of them reaches the GPU."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


def empty(*size, dtype=torch.bfloat16):
    return torch.empty(size, dtype=dtype, device="cuda")


@pytest.mark.parametrize("D", [0, 12, 264, 2 ** 32, 2 ** 32 + 8, 2 ** 40 + 128])
def test_head_sizes(ops, D):
    # also those whose low 32 bits would do
    from paper_2606_10440_amd import SimError
    cache = ops.PagedCache(empty(0, 1, 1, D), empty(0, 1, 1, D))
    with pytest.raises(SimError, match="D must be"):
        ops.cache_append(cache, empty(0, 1, D), empty(0, 1, D), empty(0, dtype=torch.int64))
    with pytest.raises(SimError, match="D must be"):
        ops.cache_attention(empty(0, 1, D), cache, empty(0, 3, dtype=torch.int32), empty(0, dtype=torch.int32))
