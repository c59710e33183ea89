"""A decode step of a layer with experts as a serving loop runs it, by the operators together: the new token's rows into the
paged cache, attention over it, the router's choice, the experts' shares of two ranks, and the next token; step by step
against 64 bits, over several steps, eagerly and from one graph."""
from __future__ import annotations

import numpy as np
import pytest

from tests import cache_reference, ops_reference, route_reference, sample_reference
from tests.test_gpu_experts import reference as experts_reference

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

B, Hq, Hkv, D, PAGE, E, K, F, V = 5, 4, 2, 64, 16, 16, 3, 96, 501
HIDDEN = Hq * D
ROUTE = dict(score="sigmoid", groups=4, top_groups=2, group_best=2, scale=2.5)


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


class Layer:
    def __init__(self, ops):
        g = torch.Generator().manual_seed(1)

        def weight(*shape):
            return (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).to(torch.bfloat16).cuda()

        self.qkv = ops.mx4_quantize(weight((Hq + 2 * Hkv) * D, HIDDEN))
        self.router = ops.mx4_quantize(weight(E, HIDDEN))
        self.head = ops.mx4_quantize(weight(V, HIDDEN))
        self.w13, self.w2 = weight(E, 2 * F, HIDDEN), weight(E, HIDDEN, F)
        self.bias = (torch.randn(E, generator=g) * 0.1).cuda()
        self.embedding = weight(V, HIDDEN)
        self.embedding *= 8
        pages = torch.randperm(B * 6, generator=g).int().cuda()
        self.table = pages.reshape(B, 6)
        self.cache = ops.PagedCache(*(torch.full((B * 6, Hkv, PAGE, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"))


def step(ops, m, x, lengths, u, seen=None):
    """x [B, hidden] of the new tokens, lengths with them: the next tokens."""
    def keep(**values):
        if seen is not None:
            seen.update(values)

    qkv = ops.mx4_matmul(x, m.qkv).unflatten(1, (-1, D))
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    at = (lengths - 1).long()
    slots = torch.gather(m.table, 1, (at // PAGE)[:, None])[:, 0].long() * PAGE + at % PAGE
    ops.cache_append(m.cache, k, v, slots)
    a = ops.cache_attention(q, m.cache, m.table, lengths, window=40)
    h = x + a.flatten(1)
    logits = ops.mx4_matmul(h, m.router, dtype=torch.float32)
    r = ops.moe_route(logits, K, bias=m.bias, **ROUTE)
    parts = [ops.moe_experts(h, r.experts, r.weights, m.w13[f:f + E // 2], m.w2[f:f + E // 2], first=f) for f in (0, E // 2)]
    y = h + parts[0] + parts[1]
    out = ops.mx4_matmul(y, m.head, dtype=torch.float32)
    token = ops.sample(out, u, temperature=0.9, top_k=50, top_p=0.95, min_p=0.01)
    keep(q=q, a=a, h=h, logits=logits, r=r, parts=parts, out=out, token=token)
    return token


def test_each_part_is_its_definition(ops):
    m = Layer(ops)
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    token = torch.arange(B, device="cuda").int()
    start = torch.tensor([0, 3, 0, 60, 30], device="cuda").int()  # how long each waits before it begins
    f64 = lambda t: t.detach().double().cpu().numpy()  # noqa: E731
    for s in range(70):
        active = s >= start
        lengths = torch.where(active, lengths + 1, 0)  # a sequence that has not begun has no tokens
        u = torch.rand(B, generator=torch.Generator().manual_seed(s)).cuda()
        seen = {}
        rows = torch.where(active, lengths, 1)         # and writes to a place that it will write again
        x = m.embedding[token.long()]
        token = step(ops, m, x, rows, u, seen)
        if s % 23 and s != 69:
            continue
        k64, v64 = (np.nan_to_num(f64(c)) for c in m.cache)
        out, bound, _, _ = cache_reference.attention(f64(seen["q"]), k64, v64, m.table.cpu().numpy(), rows.cpu().numpy(), "bf16", window=40)
        assert (np.abs(f64(seen["a"]) - out) <= bound).all()
        want = route_reference.route(f64(seen["logits"]), K, None, True, "sigmoid", m.bias.cpu().numpy(), 4, 2, 2, 2.5)
        assert np.array_equal(seen["r"].experts.cpu().numpy(), want[0])
        for f, y in zip((0, E // 2), seen["parts"]):
            e, bound = experts_reference(f64(seen["h"]), want[0], f64(seen["r"].weights), f64(m.w13[f:f + E // 2]), f64(m.w2[f:f + E // 2]), f, "bf16")
            assert (np.abs(f64(y) - e) <= bound).all()
        z, uu = f64(seen["out"]), u.cpu().numpy()
        assert token.tolist() == [sample_reference.sample(z[b], uu[b], 0.9, 50, 0.95, 0.01) for b in range(B)]
    assert ops_reference.UNIT["bf16"] == 2.0 ** -8


def test_a_graph_replays_the_steps(ops):
    def run(use_graph):
        m = Layer(ops)
        x, lengths, u = m.embedding[:B].clone(), torch.ones(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
        graph = None
        if use_graph:
            step(ops, m, x, lengths, u)  # nothing is loaded for the first time in the capture
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                held = step(ops, m, x, lengths, u)
        tokens, token = [], torch.arange(B, device="cuda")
        for s in range(30):
            x.copy_(m.embedding[token.long()])
            lengths.fill_(s + 1)
            u.copy_(torch.rand(B, generator=torch.Generator().manual_seed(s)))
            if graph:
                graph.replay()
                token = held.clone()
                torch.cuda.synchronize()
            else:
                token = step(ops, m, x, lengths, u)
            tokens.append(token.tolist())
        return tokens, m.cache

    want, cache = run(False)
    got, cache2 = run(True)
    assert got == want and len({t for row in want for t in row}) > 10
    assert torch.equal(cache.k.nan_to_num(), cache2.k.nan_to_num()) and torch.equal(cache.v.nan_to_num(), cache2.v.nan_to_num())
