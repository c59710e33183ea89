"""An expert-parallel step's traffic from the router's choices."""
from __future__ import annotations

import numpy as np
import pytest

import sim_inputs as si
from sim_inputs import moe


@pytest.mark.parametrize("T,E,k,p", [(1, 4, 2, 2), (7, 8, 3, 4), (16, 16, 4, 8), (33, 10, 2, 5), (0, 8, 2, 4)])
def test_moves_by_hand(T, E, k, p):
    rng = np.random.default_rng(T)
    experts = np.array([rng.permutation(E)[:k] for _ in range(T)]).reshape(T, k)
    if T > 2:
        experts[1] = -1
        experts[2, 1:] = -1
    want = []
    for t in range(T):
        here = t * p // T
        for r in sorted({int(e) * p // E for e in experts[t] if e >= 0} - {here}):
            want.append((here, r))
    home, away = moe.token_moves(experts, E, p)
    assert list(zip(home.tolist(), away.tolist())) == want
    src, dst = moe.transfers(home, away, 3)
    assert len(src) == 3 * len(want) and (src != dst).all()


def test_lines():
    assert [moe.lines_of(n) for n in (0, 1, 128, 129, 4096)] == [0, 1, 1, 2, 32]


def test_makespan_is_that_of_the_fullest_link(oracle_lib):
    # an ordered pair's lines share its link and nothing else: the last of M lines completes at M + L
    p, L = 4, 10
    w = si.full_mesh(p, b=1, L=L, cap=16)
    rng = np.random.default_rng(5)
    experts = np.array([rng.permutation(16)[:3] for _ in range(20)])
    home, away = moe.token_moves(experts, 16, p)
    src, dst = moe.transfers(home, away, 5)
    pairs = np.zeros((p, p), np.int64)
    np.add.at(pairs, (home, away), 1)
    r = oracle_lib.simulate(w.n_nodes, w.n_endpoints, w.row_ptr, w.col_idx, w.bw, w.lat, w.cap, w.arb,
                            txns=(src, dst, np.zeros(len(src) + 1, np.int64), np.zeros(0, np.int64)))
    assert r.makespan == pairs.max() * 5 + L


@pytest.mark.gpu
@pytest.mark.parametrize("wire", ["bf16", "mx4"])
def test_step_runs_together(wire):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from examples import expert_parallel as ex
    from paper_2606_10440_amd import ops
    from tests import ops_reference as ref
    T, E, k, D, F, p = 12, 8, 2, 256, 64, 4
    rng = np.random.default_rng(3)

    def bf16(*shape):
        return torch.from_numpy(rng.standard_normal(shape) * shape[-1] ** -0.5).to(torch.bfloat16)

    x, wr, w13, w2 = bf16(T, D) * 16, bf16(E, D), bf16(E, 2 * F, D), bf16(E, D, F)
    step = ex.run_step(x.cuda(), ops.mx4_quantize(wr.cuda()), w13.cuda(), w2.cuda(), k, p, wire, lat=10)
    v = x.double().numpy()
    logits = ops.mx4_matmul(x.cuda(), ops.mx4_quantize(wr.cuda()), dtype=torch.float32).double().cpu().numpy()
    want, bound = ref.product(ref.mx4_values(v), ref.mx4_values(wr.double().numpy()), "fp32")
    assert (np.abs(logits - want) <= bound).all()
    assert np.array_equal(step.experts, ref.route(logits, k, None, True)[0])
    arrived = ref.mx4_values(v) if wire == "mx4" else v
    y, bound = ref.layer(arrived, logits, w13.double().numpy(), w2.double().numpy(), k, None, True, "bf16")
    assert (np.abs(step.y.double().cpu().numpy() - y) <= bound).all()
    # lines of one ordered pair share its link and nothing else: the fullest pair ends last
    home, away = moe.token_moves(step.experts, E, p)
    pairs = np.zeros((p, p), np.int64)
    np.add.at(pairs, (home, away), 1)
    assert step.lines == (D // 2 + 127) // 128 + 1 if wire == "mx4" else step.lines == 2 * D // 128
    assert step.dispatch == pairs.max() * step.lines + 10
    assert step.combine == pairs.max() * (2 * D // 128) + 10
