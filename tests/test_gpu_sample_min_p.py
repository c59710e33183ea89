"""Min-p at its ends against the 64-bit definition: a min-p of 1 keeps every logit whose weight is 1 in 64 bits, whatever else is
asked for."""
from __future__ import annotations

import numpy as np
import pytest

from tests.test_gpu_sample import TYPES, check, rows, uniform

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# none of them; sorted; all that are above a border; a large top-k; top-p; both
OTHERS = [dict(), dict(top_k=40), dict(top_k=1500), dict(top_k=3000), dict(top_p=0.5), dict(top_k=3000, top_p=0.5), dict(top_k=40, top_p=0.5)]


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [300, 5003, 70001])
@pytest.mark.parametrize("temperature", [1.0, 1e6, 1e30, 3e38])
def test_one(ops, kind, V, temperature):
    z, v = rows(V, 4, V, kind)
    v[1] = np.round(v[1])  # many that tie with the highest
    z.copy_(torch.from_numpy(v).to(TYPES[kind]))
    for n, how in enumerate(OTHERS):
        check(ops, z, v, uniform(n, 4), temperature=temperature, min_p=1.0, **how)


@pytest.mark.parametrize("min_p", [1e-45, 1e-30, 0.999])
def test_others(ops, min_p):
    z, v = rows(3, 4, 5003, "fp32")
    for n, how in enumerate(OTHERS):
        for temperature in (0.05, 1.0, 1e30):
            check(ops, z, v, uniform(n, 4), temperature=temperature, min_p=min_p, **how)


def test_infinite_temperature(ops):
    z, v = rows(4, 2, 5003, "fp32")
    t, u = torch.full((2,), float("inf"), device="cuda"), uniform(1, 2)
    for how in (dict(min_p=1.0), dict(min_p=0.5)):
        got = ops.sample(z, torch.from_numpy(u).cuda(), temperature=t, **how).tolist()
        assert got == [int(np.float64(x) * 5003) for x in u]  # all weights are 1
