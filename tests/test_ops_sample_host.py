"""Sampling without a GPU: refusals and the workspace query."""
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


SAMPLE = [("logits", P), ("type", 0), ("B", 4), ("V", 100), ("stride", 100), ("u", P), ("t", None), ("t_all", 1.0), ("k", None), ("k_all", 0),
          ("p", None), ("p_all", 1.0), ("m", None), ("m_all", 0.0), ("tokens", P), ("ws", P), ("ws_bytes", 1 << 30)]
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change,want", [
    (dict(logits=None), INVALID), (dict(type=3), INVALID), (dict(type=-1), INVALID), (dict(B=-1), INVALID), (dict(V=0), INVALID),
    (dict(V=-1), INVALID), (dict(stride=99), INVALID), (dict(u=None), INVALID), (dict(tokens=None), INVALID), (dict(t_all=-1.0), INVALID),
    (dict(t_all=NAN), INVALID), (dict(t_all=INF), INVALID), (dict(k_all=-1), INVALID), (dict(p_all=-0.5), INVALID), (dict(p_all=1.5), INVALID),
    (dict(p_all=NAN), INVALID), (dict(m_all=-0.5), INVALID), (dict(m_all=1.5), INVALID), (dict(m_all=NAN), INVALID), (dict(logits=P + 2), INVALID),
    (dict(u=P + 2), INVALID), (dict(t=P + 1), INVALID), (dict(k=P + 2), INVALID), (dict(p=P + 2), INVALID), (dict(m=P + 3), INVALID),
    (dict(tokens=P + 2), INVALID), (dict(V=(1 << 20) + 1, stride=1 << 21), SIZE), (dict(B=1 << 30), SIZE), (dict(B=0), 0),
    (dict(B=0, logits=None, u=None, tokens=None), 0)])
def test_refusals(lib, change, want):
    assert run(lib, "sim_sample", SAMPLE, **change) == want


def test_workspace_query(lib):
    for bad in [(-1, 100), (0, 100), (4, 0), (4, -1), (4, (1 << 20) + 1), (1 << 40, 100)]:
        assert lib.sim_sample_workspace(*bad) == 0, bad


def test_workspace_is_needed(lib):
    for B, V in ((1, 1 << 20), (4, 100), (300, 50000)):
        need = lib.sim_sample_workspace(B, V)
        if need:
            assert run(lib, "sim_sample", SAMPLE, B=B, V=V, stride=V, ws=None) == INVALID
            assert run(lib, "sim_sample", SAMPLE, B=B, V=V, stride=V, ws=P + 8) == INVALID
            assert run(lib, "sim_sample", SAMPLE, B=B, V=V, stride=V, ws_bytes=need - 1) == INVALID
