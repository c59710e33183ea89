"""Workspace queries: nothing is asked for where the call would refuse the
sizes, so that a caller who allocates first is refused and not out of memory."""
from __future__ import annotations

import pytest

from tests.test_ops_host import LAYER, LGRAD, LINEAR, SIZE, lib, run  # noqa: F401 (lib: the fixture)

BIG = 1 << 30


@pytest.mark.parametrize("T,D,E,k,F", [(1024, 1 << 20, 32, 32, 1), (4, 64, 16, 2, 1 << 20), (4, 64, 16, 2, (1 << 31) - 1),
                                       (1024, 1 << 19, 1024, 32, 64), (4, 64, 2000, 2, 32), (4, 64, 16, 17, 32), (4, 64, 64, 33, 32),
                                       (1025, 64, 16, 2, 32), (0, 64, 16, 2, 32), (4, 0, 16, 2, 32), (4, 64, 16, 2, -1)])
def test_layer(lib, T, D, E, k, F):  # noqa: F811
    assert lib.sim_moe_layer_workspace(T, D, E, k, F) == 0
    st = run(lib, "sim_moe_layer", LAYER, T=T, D=D, x_stride=max(D, 1), y_stride=max(D, 1), E=E, stride=E, k=k, F=F)
    assert (st == 0) == (T == 0 or D == 0)


@pytest.mark.parametrize("T,D,E,k,F", [(1, 1, 1, 1, 0), (1, 1, 1, 1, 1), (1024, (1 << 20) - 1, 4, 4, 64), (16, 4096, 128, 8, 1280)])
def test_layer_that_is_taken(lib, T, D, E, k, F):  # noqa: F811
    n = lib.sim_moe_layer_workspace(T, D, E, k, F)
    assert n > 0
    sizes = dict(T=T, D=D, x_stride=D, y_stride=D, E=E, stride=E, k=k, F=F)
    assert run(lib, "sim_moe_layer", LAYER, ws_bytes=n - 1, **sizes) == 1


@pytest.mark.parametrize("M,N,K", [(BIG, 4, BIG), (BIG, BIG, 4), (4, BIG, BIG), (1 << 31, 4, 4), (4, 4, 1 << 31)])
def test_products(lib, M, N, K):  # noqa: F811
    assert lib.sim_mx4_linear_workspace(M, N, K) == 0 and lib.sim_mx4_linear_grad_workspace(M, N, K) == 0
    assert run(lib, "sim_mx4_linear", LINEAR, M=M, N=N, K=K, x_stride=K, stride=N) == SIZE
    assert run(lib, "sim_mx4_linear_grad", LGRAD, M=M, N=N, K=K, dy_stride=N, x_stride=K, w_stride=K, dx_stride=K, dw_stride=K) == SIZE


def test_linear_with_nothing_to_write(lib):  # noqa: F811
    assert lib.sim_mx4_linear_workspace(64, 0, 4096) == 0 and lib.sim_mx4_linear_workspace(64, 4, 4096) > 0
