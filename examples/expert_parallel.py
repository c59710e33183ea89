"""One expert-parallel step: what it computes on this GPU, and what its tokens
cost on a simulated fabric, in 16 bits and in 4.

    python examples/expert_parallel.py [--tokens 128 --experts 64 --k 6 --hidden 2048 --ffn 1408 --ranks 8 --top-ranks 3]

The router's product is a 4-bit one; ``ops.moe_route`` chooses the experts; the
tokens are put into the wire format; ``ops.moe_layer`` runs the experts on what
arrives; and the router's choices, as 128 B lines, are simulated over a full
mesh of endpoints: dispatch to the experts' endpoints and combine back (16-bit
partial results).  With ``--top-ranks`` a token may go to so many ranks only:
the router has sigmoid scores and a group of experts for each rank, and each
rank's share of the experts is computed by ``ops.moe_experts`` from its choices.
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import sim_inputs as si  # noqa: E402
from sim_inputs import moe  # noqa: E402


@dataclass
class Step:
    y: "object"            # [T, hidden] results
    experts: np.ndarray    # [T, k]
    lines: int             # a token on the wire
    dispatch: int          # cycles
    combine: int
    layer_us: float


def simulate(ranks, src, dst, lat, cap):
    """Cycles until the last line of the list has arrived."""
    from paper_2606_10440_amd import Simulator, sim
    if len(src) == 0:
        return 0
    w = si.full_mesh(ranks, b=1, L=lat, cap=cap)
    s = Simulator(w.n_nodes, w.n_endpoints, w.row_ptr, w.col_idx, w.bw, w.lat, w.cap, w.arb)
    try:
        s.load_transactions(src, dst, np.zeros(len(src) + 1, np.int64), [])
        r = s.run()
        if r.status != sim.SIM_OK:
            raise sim.SimError(r.status, "the simulation did not end")
        return int(r.makespan[0])
    finally:
        s.close()


def share(weights, rank, ranks):
    """A rank's experts of weights [experts, rows, columns], plain or in 4 bits."""
    from paper_2606_10440_amd import ops
    n, rows = weights.shape[0] // ranks, weights.shape[1]
    if not isinstance(weights, ops.Mx4):
        return weights[rank * n:(rank + 1) * n]
    at = slice(rank * n * rows, (rank + 1) * n * rows)
    return ops.Mx4(weights.codes[at], weights.scales[at], (n, *weights.shape[1:]))


def run_step(x, w_router, w13, w2, k, ranks, wire="mx4", lat=50, cap=64, top_ranks=None, bias=None):
    """x [T, hidden] bf16, w_router a 4-bit [experts, hidden], w13 and w2 the
    experts' weights as ``ops.moe_layer`` takes them.  With ``top_ranks`` the
    router keeps a token on so many ranks, with ``bias`` [experts] added to
    the scores for the choice."""
    import torch
    from paper_2606_10440_amd import ops
    T, hidden = x.shape
    n_experts = w_router.shape[0]
    logits = ops.mx4_matmul(x, w_router, dtype=torch.float32)
    if top_ranks is None:
        routes = ops.moe_route(logits, k)
    else:
        routes = ops.moe_route(logits, k, score="sigmoid", bias=bias, groups=ranks, top_groups=top_ranks, group_best=2)
    if wire == "mx4":
        sent = ops.mx4_quantize(x)
        lines = moe.lines_of_token(sent)
        arrived = ops.mx4_dequantize(sent, x.dtype)
    else:
        lines, arrived = moe.lines_of(2 * hidden), x

    def layer(out=None):
        if top_ranks is None:
            return ops.moe_layer(arrived, logits, w13, w2, k, out=out)
        parts = [ops.moe_experts(arrived, routes.experts, routes.weights, share(w13, r, ranks), share(w2, r, ranks),
                                 first=r * (n_experts // ranks)) for r in range(ranks)]
        return torch.stack(parts).float().sum(0).to(x.dtype)  # what combine brings together

    y = layer()
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    layer(y)
    end.record()
    experts = routes.experts.cpu().numpy()
    home, away = moe.token_moves(experts, n_experts, ranks)
    dispatch = simulate(ranks, *moe.transfers(home, away, lines), lat, cap)
    combine = simulate(ranks, *moe.transfers(away, home, moe.lines_of(2 * hidden)), lat, cap)
    end.synchronize()
    return Step(y, experts, lines, dispatch, combine, start.elapsed_time(end) * 1e3)


def main():
    import torch
    from paper_2606_10440_amd import ops
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--tokens", type=int, default=128)
    p.add_argument("--experts", type=int, default=64)
    p.add_argument("--k", type=int, default=6)
    p.add_argument("--hidden", type=int, default=2048)
    p.add_argument("--ffn", type=int, default=1408)
    p.add_argument("--ranks", type=int, default=8)
    p.add_argument("--top-ranks", type=int, default=None, help="ranks that a token may go to (default: any)")
    p.add_argument("--link-gbs", type=float, default=64.0, help="one link's GB/s: a line a cycle")
    a = p.parse_args()
    g = torch.Generator(device="cuda").manual_seed(0)

    def weight(*shape):
        return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(torch.bfloat16)

    x = torch.randn(a.tokens, a.hidden, generator=g, device="cuda").to(torch.bfloat16)
    w_router = ops.mx4_quantize(weight(a.experts, a.hidden))
    w13, w2 = (ops.mx4_quantize(weight(*s)) for s in ((a.experts, 2 * a.ffn, a.hidden), (a.experts, a.hidden, a.ffn)))
    cycle_us = si.LINE_BYTES / (a.link_gbs * 1e3)
    for wire in ("bf16", "mx4"):
        s = run_step(x, w_router, w13, w2, a.k, a.ranks, wire, top_ranks=a.top_ranks)
        print(f"{wire}: {s.lines} lines a token, dispatch {s.dispatch} cycles ({s.dispatch * cycle_us:.1f} us), "
              f"combine {s.combine} cycles ({s.combine * cycle_us:.1f} us), experts' layer {s.layer_us:.1f} us on this GPU")


if __name__ == "__main__":
    main()
