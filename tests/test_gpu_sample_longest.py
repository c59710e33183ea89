"""Sampling from the longest rows that the call takes, 2^20 logits, against the 64-bit definition: which token, exactly.  Weights
that are all the highest have the largest sums that there are."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_sample import TYPES, check, rows, uniform

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
V = 1 << 20


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


@pytest.mark.parametrize("kind", TYPES)
def test_equal_logits(ops, kind):
    # weights of 1: sums, borders and the places that u points at are whole numbers or products of two, exact in 64 bits
    v = np.full((2, V), -1.25)
    z = torch.from_numpy(v).to(TYPES[kind]).cuda()
    for n, how in enumerate([dict(top_p=0.5), dict(top_p=0.9), dict(top_p=0.9999999), dict(top_p=1e-6), dict(), dict(top_k=700000, top_p=0.75),
                             dict(top_k=V - 1), dict(top_k=2000, top_p=0.3), dict(top_p=0.6, min_p=1.0)]):
        check(ops, z, v, uniform(n, 2), **how)


@pytest.mark.parametrize("kind", TYPES)
def test_temperatures_that_make_all_weights_one(ops, kind):
    z, v = rows(1, 2, V, kind)
    for n, how in enumerate([dict(top_p=0.5), dict(top_p=0.9), dict(top_k=900000, top_p=0.7)]):
        check(ops, z, v, uniform(n, 2), temperature=3e38, **how)


@pytest.mark.parametrize("kind", TYPES)
def test_usual_settings(ops, kind):
    z, v = rows(2, 2, V, kind)
    for n, how in enumerate([dict(), dict(top_p=0.9), dict(top_k=50, top_p=0.95), dict(top_p=0.95, temperature=0.3), dict(min_p=0.05, top_p=0.99)]):
        check(ops, z, v, uniform(n, 2), **how)
