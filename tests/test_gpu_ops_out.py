"""``out=``: autograd learns of the write, and refuses what it would have to
differentiate."""
from __future__ import annotations

import pytest

from tests.test_gpu_ops import layer_case, ops  # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def calls(ops):  # noqa: F811
    """Each call that takes ``out``, and the sizes of its result."""
    x = torch.randn(4, 64, device="cuda").bfloat16()
    w = ops.mx4_quantize(torch.randn(64, 64, device="cuda"))
    q = ops.mx4_quantize(x)
    (lx, z, w13, w2), _ = layer_case(ops, 70, 4, 3, 64, 32, "bf16", "same")
    return {"plain": (lambda out: ops.mx4_matmul(x, w, out=out)), "stored": (lambda out: ops.mx4_matmul(q, w, out=out)),
            "layer": (lambda out: ops.moe_layer(lx, z, w13, w2, 2, out=out))}


NAMES = ["plain", "stored", "layer"]


@pytest.mark.parametrize("name", NAMES)
def test_a_write_to_what_autograd_has_saved_shows(ops, name):  # noqa: F811
    call = calls(ops)[name]
    a = torch.ones(4, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    out = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16)
    s = (a * out).sum()  # saves out for the gradient of a
    call(out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        s.backward()


@pytest.mark.parametrize("name", NAMES)
def test_a_result_that_requires_a_gradient_is_refused(ops, name):  # noqa: F811
    from paper_2606_10440_amd.sim import SimError
    call = calls(ops)[name]
    leaf = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
    for out in (leaf, leaf * 2):
        kept = out.detach().clone()
        with pytest.raises(SimError, match="gradient"):
            call(out)
        assert torch.equal(out.detach(), kept)
    with torch.no_grad():
        assert torch.equal(call(leaf), call(None) if name == "layer" else call(torch.empty_like(leaf)))


@pytest.mark.parametrize("name", NAMES)
def test_results_in_inference_mode(ops, name):  # noqa: F811
    call = calls(ops)[name]
    want = call(torch.empty(4, 64, device="cuda", dtype=torch.bfloat16))
    with torch.inference_mode():
        out = torch.empty(4, 64, device="cuda", dtype=torch.bfloat16)
        assert call(out) is out and torch.equal(out, want)
        before = torch.zeros_like(want)
        assert torch.equal(call(before), want)
    assert torch.equal(call(out), want)
