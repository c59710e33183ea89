"""The paged cache and sampling where offsets pass 31 and 32 bits."""
from __future__ import annotations

import numpy as np
import pytest

from tests import cache_reference as ref
from tests import sample_reference
from tests.test_gpu_cache import near

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


@pytest.mark.parametrize("page", [256, 250])
def test_cache_of_more_than_two_to_the_32_elements(ops, page):
    Hkv, D, Hq = 2, 128, 4
    pages = (1 << 32) // (2 * Hkv * page * D) + 40          # keys and values in one buffer: more than 2^32 elements
    both = torch.empty(pages, 2, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    cache = ops.PagedCache(both[:, 0], both[:, 1])
    assert both.numel() > 1 << 32
    g = np.random.default_rng(page)
    lengths = [3 * page + 7, 900]
    need = [-(-n // page) for n in lengths]
    at = [pages - 1, pages - 5, 0, pages // 2 + 1, pages - 3, pages // 2, 1, pages - 30]
    table = np.full((2, max(need)), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = [at.pop(0) for _ in range(n)]
    total = sum(lengths)
    k, v = (torch.from_numpy(g.standard_normal((total, Hkv, D))).to(torch.bfloat16) for _ in "kv")
    slots = np.concatenate([table[b, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page for b, n in enumerate(lengths)])
    assert slots.max() * Hkv * D * 2 > 1 << 31
    ops.cache_append(cache, k.cuda(), v.cuda(), torch.from_numpy(slots).cuda())
    q = torch.from_numpy(g.standard_normal((2, Hq, D))).to(torch.bfloat16)
    out, lse = ops.cache_attention(q.cuda(), cache, torch.from_numpy(table).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), return_lse=True)
    # the definition on a small cache that has these pages alone
    used = sorted(set(table[table >= 0].tolist()))
    small = np.array([[used.index(p) if p >= 0 else -1 for p in row] for row in table])
    k64, v64 = (c[used].double().cpu().numpy() for c in cache)
    for c in (k64, v64):
        c[~np.isfinite(c)] = 0  # places without a token
    want = ref.attention(q.double().numpy(), k64, v64, small, lengths, "bf16")
    near(out, *want[:2])
    near(lse, *want[2:])
    assert torch.equal(cache.k[table[0, 0], :, 0].cpu(), k[0])


def test_sampling_more_than_two_to_the_31_logits(ops):
    V, B = (1 << 20) - 3, 2100
    z = torch.full((B, V), -20.0, dtype=torch.float16, device="cuda")
    assert z.numel() > 1 << 31
    g = np.random.default_rng(1)
    rows = [0, 1023, 1024, 2047, 2048, B - 1]
    u = g.random(B).astype(np.float32)
    for b in rows:
        z[b] = torch.from_numpy(g.standard_normal(V) * 2).half()
    for how in (dict(top_k=40, top_p=0.9), dict(), dict(top_p=0.8)):
        got = ops.sample(z, torch.from_numpy(u).cuda(), **how).cpu().numpy()
        for b in rows:
            assert got[b] == sample_reference.sample(z[b].double().cpu().numpy(), u[b], **how)


def test_many_heads_and_no_pages(ops):
    # one unit for all sequences together where the heads alone fill the GPU
    k = torch.zeros(1, 800, 1, 8, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, 800, 8, dtype=torch.bfloat16, device="cuda")
    table = torch.full((3, 2000), -1, dtype=torch.int32, device="cuda")
    lengths = torch.tensor([2000, 5, 1999], dtype=torch.int32, device="cuda")
    out, lse = ops.cache_attention(q, ops.PagedCache(k, k.clone()), table, lengths, return_lse=True)
    assert not out.any() and (lse == float("-inf")).all()


def test_lengths_that_add_up_past_31_bits(ops):
    # 64 sequences of 2^30 tokens, 2^31 steps of 32, on pages that are not there but for one of 2^20 tokens
    page, D = 1 << 20, 8
    k = torch.zeros(1, 1, page, D, dtype=torch.bfloat16, device="cuda")
    table = torch.full((64, (1 << 30) // page), -1, dtype=torch.int32, device="cuda")
    table[5, 0] = table[63, -1] = 0
    lengths = torch.full((64,), 1 << 30, dtype=torch.int32, device="cuda")
    q = torch.ones(64, 1, D, dtype=torch.bfloat16, device="cuda")
    out, lse = ops.cache_attention(q, ops.PagedCache(k, torch.ones_like(k)), table, lengths, return_lse=True)
    some = torch.zeros(64, dtype=torch.bool)
    some[[5, 63]] = True
    out, lse = out.cpu().float(), lse.cpu()
    assert (out[some] == 1).all() and not out[~some].any()  # sums of ones up to 2^20 are exact
    assert (lse[~some] == float("-inf")).all()
    assert ((lse[some].double() - 20 * np.log(2)).abs() <= 4 * 20 * np.log(2) * 2.0 ** -24).all()  # a logarithm, a constant, a product
