"""Attention over the cache where scores are so large that 32 bits hold them to whole numbers only: weights go by the scores'
differences."""
from __future__ import annotations

import numpy as np
import pytest

from tests import cache_reference as ref
from tests.test_gpu_cache import TYPES, Case, attend, near

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
LN2 = float(np.float32(np.log(2.0)))  # times log2 e it is 1 in 32 bits: a score is the power of two that its weight is


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("power", [0, 20, 23, 24, 25, 26])
@pytest.mark.parametrize("n", [1, 100, 700, 3000])
def test_weights_go_by_differences(ops, kind, sign, power, n):
    # a score is +-2^power and 8 times a whole number, which is exact up to 2^27
    c = Case(ops, [n, n], kind, Hq=2, Hkv=1, D=64, page=16, seed=power)
    g = np.random.default_rng(n)
    q, k = np.zeros((2, 2, 64)), np.zeros(c.k64.shape)
    q[..., 0], q[..., 1] = sign * 2.0 ** (power // 2), 2.0
    add = -g.integers(0, 4, (2, n))
    for b in range(2):
        for j in range(n):
            k[c.table[b, j // 16], 0, j % 16, :2] = 2.0 ** (power - power // 2), 4.0 * add[b, j]
    c.q.copy_(torch.from_numpy(q))
    c.cache.k.copy_(torch.from_numpy(k))
    out, lse = attend(ops, c, scale=LN2)
    v = [np.stack([c.v64[c.table[b, j // 16], 0, j % 16] for j in range(n)]) for b in range(2)]
    p = [2.0 ** (8.0 * (a - a.max())) for a in add]
    want = np.stack([np.repeat((w @ x / w.sum())[None], 2, 0) for w, x in zip(p, v)])
    size = np.stack([np.repeat((w @ np.abs(x) / w.sum())[None], 2, 0) for w, x in zip(p, v)])
    # the weights are exact but for a 2^x of 32 bits; sums of n terms, the cuts' and the waves' joints; one rounding
    rel = ref.PARTS[kind] + (n + 64) * ref.U32
    near(out, want, rel * size + ref.UNIT[kind] * (np.abs(want) + rel * size) + ref.TINY[kind] + n * 2.0 ** -38 * np.abs(v[0]).max())
    total = np.array([8.0 * a.max() + sign * 2.0 ** power + np.log2(w.sum()) for a, w in zip(add, p)]) * np.log(2.0)
    near(lse, np.repeat(total[:, None], 2, 1), 4 * ref.U32 * np.abs(total)[:, None] + (n + 64) * ref.U32 + 2.0 ** -22)
