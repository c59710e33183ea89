"""What a token takes on the wire, at hidden sizes that are no multiple of a line."""
from __future__ import annotations

from collections import namedtuple

import numpy as np
import pytest

from sim_inputs import moe
from tests import ops_reference as ref

Stored = namedtuple("Stored", "codes scales")


@pytest.mark.parametrize("hidden,codes,scales", [(1, 1, 1), (255, 1, 1), (256, 1, 1), (257, 2, 1), (2048, 8, 1), (4096, 16, 1),
                                                 (4097, 17, 2), (8192, 32, 2), (8193, 33, 3)])
def test_lines_of_a_stored_token(hidden, codes, scales):
    q = Stored(*ref.mx4_stored(np.ones((1, hidden))))
    assert moe.lines_of_token(q) == codes + scales
    # the padding of a stored row is never a line of its own
    assert moe.lines_of_token(q) == moe.lines_of(-(-hidden // 2)) + moe.lines_of(-(-hidden // 32))


@pytest.mark.gpu
def test_step_of_an_odd_hidden_size():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from examples import expert_parallel as ex
    from paper_2606_10440_amd import ops
    T, E, D, F, p = 12, 8, 257, 64, 4
    g = torch.Generator(device="cuda").manual_seed(1)

    def bf16(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)

    step = ex.run_step(bf16(T, D), ops.mx4_quantize(bf16(E, D)), bf16(E, 2 * F, D), bf16(E, D, F), 2, p, "mx4", lat=10)
    home, away = moe.token_moves(step.experts, E, p)
    pairs = np.zeros((p, p), np.int64)
    np.add.at(pairs, (home, away), 1)
    assert step.lines == 3 and step.dispatch == pairs.max() * 3 + 10
