"""The experts' layer on given choices on the GPU against its 64-bit definition: each of its forms, shares of the experts,
choices outside the share or named twice, strides, graphs."""
from __future__ import annotations

import numpy as np
import pytest

from tests import ops_reference as base

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
U32 = base.U32


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


def reference(x, experts, weights, w13, w2, first, kind):
    """(y, bound): 32-bit sums of D and F products, 16 bits kept of the hidden values, one rounding."""
    T, D = x.shape
    n, _, F = w2.shape
    y, err = np.zeros((T, D)), np.zeros((T, D))
    for t in range(T):
        for e in {int(e) for e in experts[t]}:
            if not first <= e < first + n:
                continue
            named = experts[t] == e
            w, size_w = weights[t][named].sum(), np.abs(weights[t][named]).sum()
            a, b = w13[e - first], w2[e - first]
            gu, size = a @ x[t], np.abs(a) @ np.abs(x[t])
            dgu = (D + 8) * U32 * size
            sg = gu[:F] / (1 + np.exp(-gu[:F]))
            h = sg * gu[F:] * w
            dh = size_w * (1.1 * dgu[:F] * np.abs(gu[F:]) + np.abs(sg) * dgu[F:] + 1.1 * dgu[:F] * dgu[F:])
            dh += np.abs(sg * gu[F:]) * size_w * (2.0 ** -16 + (16 + named.sum()) * U32) + size_w * np.abs(gu[F:]) * 2.0 ** -120
            y[t] += b @ h
            err[t] += np.abs(b) @ dh + (F + len(experts[t]) + 8) * U32 * (np.abs(b) @ np.abs(h))
    return y, err + base.UNIT[kind] * (np.abs(y) + err) + base.TINY[kind]


def make(ops, seed, T, E, n, first, k, D, F, kind, weights, pad=0):
    g = np.random.default_rng(seed)
    t = TYPES[kind]
    x = torch.full((T, D + pad), float("nan"), dtype=t)
    x[:, :D] = torch.from_numpy(g.standard_normal((T, D))).to(t)
    x = x.cuda()[:, :D]
    experts = np.stack([g.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    share = (g.random((T, k)) - 0.2).astype(np.float32)
    w = []
    for shape in ((n, 2 * F, D), (n, D, F)):
        v = torch.from_numpy(g.standard_normal(shape) * shape[-1] ** -0.5).to(t).cuda()
        if weights == "mx4":
            v = ops.mx4_quantize(v)
            w.append((v, ops.mx4_dequantize(v, torch.float32).double().cpu().numpy()))
        else:
            w.append((v, v.double().cpu().numpy()))
    return x, experts, share, w


def run(ops, x, experts, share, w, first, **how):
    return ops.moe_experts(x, torch.from_numpy(experts).cuda(), torch.from_numpy(share).cuda(), w[0][0], w[1][0], first=first, **how)


def check(y, x, experts, share, w, first, kind):
    want, bound = reference(x.double().cpu().numpy(), experts, share.astype(np.float64), w[0][1], w[1][1], first, kind)
    off = np.abs(y.double().cpu().numpy() - want)
    assert (off <= bound).all(), float((off - bound).max())


# T, E, n, first, k, D, F: few tokens, lists of one, two and four tiles, tiny rows
CASES = [(1, 8, 8, 0, 2, 64, 32), (1, 64, 4, 60, 6, 256, 96), (3, 4, 1, 2, 4, 200, 40), (16, 32, 8, 8, 3, 384, 130), (16, 300, 290, 5, 8, 64, 64),
         (7, 12, 5, 0, 5, 4, 6), (17, 16, 4, 4, 4, 128, 64), (64, 8, 8, 0, 3, 256, 64), (65, 64, 16, 16, 8, 256, 100), (130, 4, 4, 0, 2, 256, 512),
         (200, 3, 2, 1, 3, 136, 272), (300, 600, 600, 0, 6, 64, 32), (1024, 16, 2, 7, 1, 64, 32)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("weights", ["same", "mx4"])
@pytest.mark.parametrize("case", CASES)
def test_layer(ops, kind, weights, case):
    T, E, n, first, k, D, F = case
    c = make(ops, T + E, T, E, n, first, k, D, F, kind, weights, pad=3 if T % 2 else 0)
    y = run(ops, *c, first)
    check(y, *c, first, kind)
    assert torch.equal(y, run(ops, *c, first))


@pytest.mark.parametrize("weights", ["same", "mx4"])
@pytest.mark.parametrize("T", [5, 16, 40, 90])
def test_choices_outside_and_named_twice(ops, weights, T):
    E, n, first, k, D, F = 12, 6, 3, 20, 128, 64
    x, experts, share, w = make(ops, T, T, E, n, first, 12, D, F, "bf16", weights)
    g = np.random.default_rng(1)
    experts = g.integers(0, E, (T, k)).astype(np.int32)           # many twice or more
    share = g.random((T, k)).astype(np.float32)
    experts[0] = -1                                               # a token without experts
    experts[1] = [np.iinfo(np.int32).min, np.iinfo(np.int32).max, -1, first + n, first - 1] * 4
    experts[2] = first                                            # one alone, twenty times
    experts[3, 5:] = -1
    y = run(ops, x, experts, share, w, first)
    check(y, x, experts, share, w, first, "bf16")
    assert not y[0].any() and not y[1].any()


def test_a_share_that_no_token_chose(ops):
    for T in (4, 50):
        x, experts, share, w = make(ops, 1, T, 8, 4, 0, 2, 64, 32, "bf16", "same")
        y = run(ops, x, experts + 4, share, w, 0)
        assert not run(ops, x, np.full_like(experts, 100), share, w, 0).any()
        check(y, x, experts + 4, share, w, 0, "bf16")


@pytest.mark.parametrize("T", [2, 16, 100])
@pytest.mark.parametrize("weights", ["same", "mx4"])
def test_shares_add_up_to_the_layer(ops, T, weights):
    """A router with sigmoid scores and groups, four ranks' shares of its experts, and the sum of what they give."""
    E, k, D, F = 32, 4, 256, 128
    x, _, _, w = make(ops, 3, T, E, E, 0, k, D, F, "bf16", weights)
    z = torch.randn(T, E, generator=torch.Generator().manual_seed(T)).cuda()
    bias = torch.linspace(-0.1, 0.1, E, device="cuda")
    r = ops.moe_route(z, k, score="sigmoid", bias=bias, groups=8, top_groups=4, group_best=2, scale=2.5)
    whole = ops.moe_experts(x, r.experts, r.weights, w[0][0], w[1][0])
    args = (x, r.experts.cpu().numpy(), r.weights.cpu().numpy())
    check(whole, *args, w, 0, "bf16")

    def part(v, rows, rank):
        if weights != "mx4":
            return v[rank * 8:rank * 8 + 8]
        at = slice(rank * 8 * rows, (rank + 1) * 8 * rows)
        return ops.Mx4(v.codes[at], v.scales[at], (8, rows, v.shape[2]))

    total = torch.zeros(T, D, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    for rank in range(4):
        y = ops.moe_experts(x, r.experts, r.weights, part(w[0][0], 2 * F, rank), part(w[1][0], D, rank), first=rank * 8)
        total += y.double()
        size += y.double().abs()
    want, bound = reference(x.double().cpu().numpy(), *args[1:], w[0][1], w[1][1], 0, "bf16")
    # each share's result is rounded by itself
    assert (np.abs(total.cpu().numpy() - want) <= bound + (base.UNIT["bf16"] * size).cpu().numpy()).all()


def test_as_the_layer_that_routes_by_itself(ops):
    for T in (6, 48):
        x, _, _, w = make(ops, 4, T, 16, 16, 0, 3, 128, 64, "bf16", "same")
        z = torch.randn(T, 16, generator=torch.Generator().manual_seed(T)).cuda()
        r = ops.moe_route(z, 3)
        a, b = ops.moe_experts(x, r.experts, r.weights, w[0][0], w[1][0]), ops.moe_layer(x, z, w[0][0], w[1][0], 3)
        # the weights of the two agree to a few units in the last place; each result is rounded once
        assert ((a.double() - b.double()).abs() <= 2 * base.UNIT["bf16"] * a.double().abs() + 1e-4).all()


@pytest.mark.parametrize("T", [9, 70])
def test_in_place_streams_and_graph(ops, T):
    x, experts, share, w = make(ops, 5, T, 16, 8, 4, 4, 128, 64, "bf16", "same")
    want = run(ops, x, experts, share, w, 4)
    y = x.clone()
    assert run(ops, y, experts, share, w, 4, out=y) is y and torch.equal(y, want)
    de, ds = torch.from_numpy(experts).cuda(), torch.from_numpy(share).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.moe_experts(x, de, ds, w[0][0], w[1][0], first=4)
    side.synchronize()
    assert torch.equal(got, want)
    held = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.moe_experts(held, de, ds, w[0][0], w[1][0], first=4)
    for i in range(4):
        v = torch.randn(T, 128, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda()
        held.copy_(v)
        graph.replay()
        want = ops.moe_experts(v, de, ds, w[0][0], w[1][0], first=4)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals(ops):
    from paper_2606_10440_amd import SimError
    x, experts, share, w = make(ops, 6, 4, 8, 8, 0, 2, 64, 32, "bf16", "same")
    e, s = torch.from_numpy(experts).cuda(), torch.from_numpy(share).cuda()
    good = dict(x=x, experts=e, weights=s, w13=w[0][0], w2=w[1][0])
    for bad in [dict(x=x.float()), dict(x=x.half()), dict(x=x[0]), dict(experts=e.long()), dict(experts=e[:3]), dict(experts=e[:, :1]),
                dict(weights=s.double()), dict(weights=s.t().contiguous().t()), dict(experts=e.cpu()), dict(w13=w[0][0][:4]), dict(w2=w[1][0].float()),
                dict(w13=w[0][0].cpu()), dict(w2=w[1][0][:, :32]), dict(first=-1), dict(first=2 ** 31 - 4), dict(first=2 ** 40), dict(out=x.float()),
                dict(out=torch.empty_like(x).requires_grad_()), dict(experts=e[:, :0], weights=s[:, :0]),
                dict(experts=e.repeat(1, 20), weights=s.repeat(1, 20)), dict(w13=w[0][0][:0], w2=w[1][0][:0])]:
        with pytest.raises(SimError):
            ops.moe_experts(**{**good, **bad})
    big = x[:1].expand(1025, -1).contiguous()
    with pytest.raises(SimError):
        ops.moe_experts(big, e[:1].expand(1025, -1).contiguous(), s[:1].expand(1025, -1).contiguous(), w[0][0], w[1][0])
    assert ops.moe_experts(x[:0], e[:0], s[:0], w[0][0], w[1][0]).shape == (0, 64)
