"""The router with scores without a GPU: its refusals."""
from __future__ import annotations

import os

import pytest

from tests.test_ops_host import INVALID, P, ROUTE, ROUTE_BAD, run


@pytest.fixture(scope="module")
def lib():
    from paper_2606_10440_amd import ops, sim
    if not os.path.exists(sim.LIB_PATH):
        from paper_2606_10440_amd import build
        build.build()
    return ops.lib()


SCORED = ROUTE[:7] + [("score", 1), ("bias", None), ("groups", 4), ("top_groups", 2), ("best", 2), ("k", 2), ("renorm", 1),
                      ("scale", 1.0)] + ROUTE[9:]
ODD = [(dict(score=2), INVALID), (dict(score=-1), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=-float("inf")), INVALID)]


@pytest.mark.parametrize("change,want", ROUTE_BAD + ODD + [
    (dict(bias=P + 2), INVALID), (dict(groups=0), INVALID), (dict(groups=3), INVALID), (dict(groups=32), INVALID), (dict(groups=-4), INVALID),
    (dict(E=256, stride=256, groups=128), INVALID), (dict(top_groups=0), INVALID), (dict(top_groups=5), INVALID), (dict(best=0), INVALID),
    (dict(best=3), INVALID), (dict(experts=None), INVALID), (dict(weights=None), INVALID), (dict(order=None), INVALID),
    (dict(offsets=None), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=0), INVALID), (dict(weights=P + 1), INVALID)])
def test_refusals(lib, change, want):
    assert run(lib, "sim_moe_route_scored", SCORED, **change) == want


GRAD = ROUTE[:7] + [("score", 1), ("k", 2), ("renorm", 1), ("scale", 1.0), ("experts", P), ("dw", P), ("dz", P)]


@pytest.mark.parametrize("change,want", ROUTE_BAD + ODD + [
    (dict(experts=None), INVALID), (dict(dw=None), INVALID), (dict(dz=None), INVALID), (dict(dz=P + 2), INVALID), (dict(T=0), 0)])
def test_gradient_refusals(lib, change, want):
    assert run(lib, "sim_moe_route_scored_grad", GRAD, **change) == want
