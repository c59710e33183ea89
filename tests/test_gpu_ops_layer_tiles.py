"""The experts' layer where each of its tilings for long lists is taken: one,
two and four column tiles, lists of one workgroup and shared ones, whole rows
and rows with an end, on lists of even and of very different lengths."""
from __future__ import annotations

import pytest

from tests import ops_reference as ref
from tests.test_gpu_ops import check, layer_case, masks, ops  # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# T, E, k, D, F
CASES = [(40, 9, 3, 128, 256), (40, 9, 3, 136, 260), (130, 5, 2, 192, 320), (130, 5, 2, 100, 330),   # two
         (100, 9, 3, 64, 960), (100, 9, 3, 72, 964), (150, 3, 2, 65, 33), (200, 4, 2, 65, 128),      # four
         (60, 4, 2, 256, 64), (130, 3, 2, 128, 96), (300, 8, 1, 64, 40)]                             # one


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("weights", ["same", "mx4"])
@pytest.mark.parametrize("case", CASES)
@pytest.mark.parametrize("how", ["none", "expert", "token", "one"])
def test_layer(ops, kind, weights, case, how):  # noqa: F811
    T, E, k, D, F = case
    (x, z, w13, w2), (vx, vz, v13, v2) = layer_case(ops, 60, T, E, D, F, kind, weights)
    if how == "one":  # nearly all tokens want the last expert first
        z[:-3, -1] += 64
        m = None
    else:
        m = masks(T, E, how, seed=T)
    # ties or rounding must not decide what is compared: the reference reads what the kernel reads
    vz = z.double().cpu().numpy()
    got = ops.moe_layer(x, z, w13, w2, k, mask=None if m is None else torch.from_numpy(m).cuda(), renormalize=T % 3 != 0)
    check(got, *ref.layer(vx, vz, v13, v2, k, m, T % 3 != 0, kind))
