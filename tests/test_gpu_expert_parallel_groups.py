"""The expert-parallel example with a router that keeps a token on few ranks: what it computes and what it sends."""
from __future__ import annotations

import numpy as np
import pytest

from sim_inputs import moe
from tests.test_gpu_experts import reference

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("weights", ["bf16", "mx4"])
def test_few_ranks(weights):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from examples import expert_parallel as ex
    from paper_2606_10440_amd import ops
    T, E, D, F, p, k, top = 48, 16, 256, 64, 4, 4, 2
    g = torch.Generator(device="cuda").manual_seed(1)

    def bf16(*shape):
        return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).to(torch.bfloat16)

    x, router, w13, w2 = bf16(T, D) * 16, ops.mx4_quantize(bf16(E, D)), bf16(E, 2 * F, D), bf16(E, D, F)
    if weights == "mx4":
        w13, w2 = ops.mx4_quantize(w13), ops.mx4_quantize(w2)
    bias = torch.linspace(-0.1, 0.1, E, device="cuda")
    step = ex.run_step(x, router, w13, w2, k, p, "bf16", lat=10, top_ranks=top, bias=bias)
    owner = step.experts * p // E
    assert max(len(set(row)) for row in owner.tolist()) <= top
    home, away = moe.token_moves(step.experts, E, p)
    pairs = np.zeros((p, p), np.int64)
    np.add.at(pairs, (home, away), 1)
    assert step.dispatch == pairs.max() * step.lines + 10
    logits = ops.mx4_matmul(x, router, dtype=torch.float32)
    r = ops.moe_route(logits, k, score="sigmoid", bias=bias, groups=p, top_groups=top, group_best=2)
    assert np.array_equal(r.experts.cpu().numpy(), step.experts)
    w = [(ops.mx4_dequantize(v, torch.float32) if weights == "mx4" else v).double().cpu().numpy() for v in (w13, w2)]
    args = (x.double().cpu().numpy(), step.experts, r.weights.double().cpu().numpy())
    want, bound = reference(*args, *w, 0, "bf16")
    # each rank's part is rounded by itself before they are added
    parts = sum(np.abs(reference(*args, w[0][f:f + 4], w[1][f:f + 4], f, "bf16")[0]) for f in range(0, E, 4))
    assert (np.abs(step.y.double().cpu().numpy() - want) <= 2 * bound + 2.0 ** -8 * parts).all()
