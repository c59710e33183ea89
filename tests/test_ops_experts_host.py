"""The experts' layer on given choices without a GPU: refusals and the workspace query."""
from __future__ import annotations

import os

import pytest

from tests.test_ops_host import INVALID, P, SIZE, run


@pytest.fixture(scope="module")
def lib():
    from paper_2606_10440_amd import ops, sim
    if not os.path.exists(sim.LIB_PATH):
        from paper_2606_10440_amd import build
        build.build()
    return ops.lib()


EXPERTS = [("x", P), ("type", 2), ("T", 4), ("D", 64), ("x_stride", 64), ("experts", P), ("weights", P), ("k", 2), ("first", 8), ("n", 16),
           ("w13", P), ("s13", None), ("w2", P), ("s2", None), ("weight_type", 2), ("F", 32), ("y", P), ("y_stride", 64), ("ws", P),
           ("ws_bytes", 1 << 30)]


@pytest.mark.parametrize("change,want", [
    (dict(x=None), INVALID), (dict(type=0, weight_type=0), INVALID), (dict(weight_type=1), INVALID), (dict(weight_type=3), INVALID),
    (dict(s13=P), INVALID), (dict(w2=None), INVALID), (dict(w13=None), INVALID), (dict(experts=None), INVALID), (dict(weights=None), INVALID),
    (dict(y=None), INVALID), (dict(k=0), INVALID), (dict(k=33), INVALID), (dict(n=0), INVALID), (dict(n=1025), INVALID),
    (dict(first=-1), INVALID), (dict(first=(1 << 31) - 8), INVALID), (dict(T=-1), INVALID), (dict(F=-1), INVALID), (dict(T=1025), SIZE),
    (dict(D=1 << 20), SIZE), (dict(F=1 << 20), SIZE), (dict(x_stride=63), INVALID), (dict(y_stride=63), INVALID), (dict(ws=None), INVALID),
    (dict(ws_bytes=100), INVALID), (dict(ws=P + 8), INVALID), (dict(experts=P + 2), INVALID), (dict(weights=P + 1), INVALID),
    (dict(w13=P + 1), INVALID), (dict(T=0), 0), (dict(D=0), 0)])
def test_refusals(lib, change, want):
    assert run(lib, "sim_moe_experts", EXPERTS, **change) == want


def test_workspace_query(lib):
    ask = lib.sim_moe_experts_workspace
    for bad in [(0, 64, 16, 2, 32), (-1, 64, 16, 2, 32), (1025, 64, 16, 2, 32), (4, 0, 16, 2, 32), (4, 64, 0, 2, 32), (4, 64, 1025, 2, 32),
                (4, 64, 16, 0, 32), (4, 64, 16, 33, 32), (4, 64, 16, 2, -1), (4, 1 << 20, 16, 2, 32), (4, 64, 16, 2, 1 << 31)]:
        assert ask(*bad) == 0, bad
    assert ask(4, 64, 1, 20, 32) > 0  # more choices than experts in the share
