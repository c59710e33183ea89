"""Calls on the paged cache that are refused before anything reaches the GPU, and those next to them that are not."""
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


def test_parts_that_share_memory(ops):
    from paper_2606_10440_amd import SimError
    pages, Hkv, page, D = 6, 2, 16, 64
    rows = torch.zeros(2, Hkv, D, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([3, 40], device="cuda")
    one = empty(pages, 2, Hkv, page, D).zero_()
    flat = one.reshape(pages * 2, Hkv, page, D)

    def part(first, stride=2, n=pages - 1):
        return flat[first:][::stride][:n]

    for k, v in [(part(0), part(0)), (part(0), part(2)), (part(1), part(5)), (part(0, 1), part(1, 1)), (part(0), part(1, 1)),
                 (one[:, 0], flat.flatten()[64:64 + pages * flat[0].numel()].view(pages, Hkv, page, D))]:
        with pytest.raises(SimError, match="own"):
            ops.cache_append(ops.PagedCache(k[:min(len(k), len(v))], v[:min(len(k), len(v))]), rows, rows, slots)
    assert not one.any()
    for k, v in [(one[:, 0], one[:, 1]), (one[:, 1], one[:, 0]), (flat[:6], flat[6:]), (part(0), part(3)), (flat[6:7], flat[5:6])]:
        cache = ops.PagedCache(k, v)
        at = torch.tensor([3, 12], device="cuda")
        ops.cache_append(cache, rows + 1, rows + 2, at)
        assert (k[0, :, [3, 12]] == 1).all() and (v[0, :, [3, 12]] == 2).all()
        assert one.sum() == 3 * rows.numel()
        one.zero_()


def test_rows_of_the_cache_itself(ops):
    # a page is copied to another one, as where two sequences part
    pages, Hkv, page, D = 6, 2, 16, 64
    one = torch.randn(pages, 2, Hkv, page, D, device="cuda").to(torch.bfloat16)
    cache = ops.PagedCache(one[:, 0], one[:, 1])
    want = one.clone()
    want[4, :, :, :11] = want[1, :, :, :11]
    k, v = (c[1, :, :11].transpose(0, 1) for c in cache)
    ops.cache_append(cache, k, v, 4 * page + torch.arange(11, device="cuda"))
    assert torch.equal(one, want)
