"""The router's gradient for tokens that have few experts to choose from or
none: logits of -infinity in the place of a mask, rows of the type's lowest
value, fewer experts than choices.  Bounds are those of ``ops_reference``."""
from __future__ import annotations

import numpy as np
import pytest

from tests import ops_reference as ref
from tests.test_gpu_ops import TYPES, check, check_route, ops  # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
INF = float("inf")


def rows(E, kind):
    """Logits of one row of each sort, E of them; the first is ordinary."""
    low = float(torch.finfo(TYPES[kind]).min)
    rng = np.random.default_rng(E)
    v = rng.standard_normal((7, E)) * 1.5
    v[1] = -INF
    v[2], v[2, E - 1] = -INF, 0.5      # one expert left, the last
    v[3, ::2] = -INF
    v[4] = low
    v[5], v[5, 0] = -INF, low          # the lowest value is a logit like any other
    v[6, 1:] = low
    z = torch.from_numpy(v).to(TYPES[kind])
    return z.cuda(), z.double().numpy()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("E,k", [(1, 1), (6, 4), (16, 16), (17, 3), (64, 8), (100, 32), (300, 5), (1000, 10)])
@pytest.mark.parametrize("how", ["none", "one", "token"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_where_few_or_no_experts_are_left(ops, kind, E, k, how, renorm):  # noqa: F811
    z, v = rows(E, kind)
    m = None
    if how == "one":      # the same for all tokens: some rows lose what -infinity had left them
        m = np.arange(E) < max(1, E - 1)
    elif how == "token":
        m = np.random.default_rng(E + 1).random((len(v), E)) < 0.5
        m[0] = False
    dm = None if m is None else torch.from_numpy(m).cuda()
    want = ref.route(v, k, m, renorm)
    r = ops.moe_route(z, k, mask=dm, renormalize=renorm)
    check_route(r, want)
    g = np.random.default_rng(2).standard_normal((len(v), k)).astype(np.float32)
    g[want[0] < 0] = np.nan  # what stands beside a choice of -1 has no effect
    dz = ops.moe_route_grad(z, r.experts, torch.from_numpy(g).cuda(), mask=dm, renormalize=renorm)
    wz, bound = ref.route_grad(v, want[0], g.astype(np.float64), m, renorm)
    check(dz, wz, bound + ref.UNIT[kind] * (np.abs(wz) + bound) + ref.TINY[kind])


@pytest.mark.parametrize("renorm", [True, False])
def test_training_step_with_a_dropped_token(ops, renorm):  # noqa: F811
    # a padded token dropped by -infinity gives no gradient and leaves the router's weights finite
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(9, 32, generator=g, device="cuda")
    w = torch.randn(12, 32, generator=g, device="cuda").requires_grad_()
    pad = torch.zeros(9, 1, dtype=torch.bool, device="cuda")
    pad[4] = True
    z = (x @ w.t()).masked_fill(pad, -INF)
    z.retain_grad()
    r = ops.moe_route_train(z, 3, renormalize=renorm)
    (r.weights * torch.arange(1.0, 4.0, device="cuda")).sum().backward()
    assert (r.experts[4] == -1).all() and (z.grad[4] == 0).all()
    assert torch.isfinite(w.grad).all() and (w.grad != 0).any()


@pytest.mark.parametrize("E,k", [(2, 1), (9, 1), (16, 1), (16, 2), (16, 15), (32, 1), (33, 16), (33, 17)])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_of_experts_held_by_other_lanes_than_the_choice(ops, E, k, renorm):  # noqa: F811
    # token t's highest logit is expert t's: a choice is handed from the lane of its place to the lane of its expert
    v = np.random.default_rng(E).permutation(E * E).reshape(E, E) / float(E * E)
    v[np.arange(E), np.arange(E)] = 2.0
    z = torch.from_numpy(v).float().cuda()
    v = z.double().cpu().numpy()
    want = ref.route(v, k, None, renorm)
    r = ops.moe_route(z, k, renormalize=renorm)
    check_route(r, want)
    g = np.random.default_rng(3).standard_normal((E, k)).astype(np.float32)
    dz = ops.moe_route_grad(z, r.experts, torch.from_numpy(g).cuda(), renormalize=renorm)
    wz, bound = ref.route_grad(v, want[0], g.astype(np.float64), None, renorm)
    check(dz, wz, bound + ref.UNIT["fp32"] * (np.abs(wz) + bound) + ref.TINY["fp32"])
