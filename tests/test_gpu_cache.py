"""The paged cache on the GPU against its 64-bit definition: lengths from nothing to many units, page sizes that end inside
a step, head sizes and groups of every form, windows, missing pages, what lies in places that are not read, strides, graphs."""
from __future__ import annotations

import numpy as np
import pytest

from tests import cache_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


class Case:
    """A cache with NaN wherever no token lies, tables of garbage behind the sequences' pages."""

    def __init__(self, ops, lengths, kind="bf16", Hq=8, Hkv=2, D=128, page=16, seed=0, spread=1.0, both=False, extra=0):
        g = np.random.default_rng(seed)
        need = [-(-max(n, 0) // page) for n in lengths]
        pages = sum(need) + 2
        order = g.permutation(pages)
        self.table = g.integers(-5, pages + 5, (len(lengths), max(need + [1]) + extra)).astype(np.int32)
        k, v = (np.full((pages, Hkv, page, D), np.nan) for _ in "kv")
        at = 0
        for b, n in enumerate(lengths):
            self.table[b, :need[b]] = order[at:at + need[b]]
            for j in range(n):
                p = self.table[b, j // page]
                k[p, :, j % page], v[p, :, j % page] = g.standard_normal((2, Hkv, D))
            at += need[b]
        q = g.standard_normal((len(lengths), Hq, D)) * spread
        t = TYPES[kind]
        self.q, kk, vv = (torch.from_numpy(x).to(t) for x in (q, k, v))
        self.q64, self.k64, self.v64 = (x.double().numpy() for x in (self.q, kk, vv))
        if both:  # keys and values as parts of one buffer
            one = torch.stack((kk, vv), 1).cuda()
            self.cache = ops.PagedCache(one[:, 0], one[:, 1])
        else:
            self.cache = ops.PagedCache(kk.cuda(), vv.cuda())
        self.q, self.kind, self.lengths = self.q.cuda(), kind, np.array(lengths, np.int32)
        self.dtable, self.dlengths = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lengths).cuda()

    def want(self, **how):
        return ref.attention(self.q64, self.k64, self.v64, self.table, self.lengths, self.kind, **how)

    def check(self, got, **how):
        out, bound, lse, lse_bound = self.want(**how)
        near(got[0], out, bound)
        near(got[1], lse, lse_bound)


def near(got, want, bound):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    same = (got == want) | np.isnan(want)
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want))
        over = off - np.where(same, 0.0, bound)
    assert not (over > 0).any(), (np.unravel_index(np.argmax(over), off.shape), float(off.max()), float(over.max()))


def attend(ops, c, **how):
    return ops.cache_attention(c.q, c.cache, c.dtable, c.dlengths, return_lse=True, **how)


LENGTHS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 0, 517]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("page", [1, 3, 16, 24, 32, 48, 128, 1000])
def test_lengths_and_pages(ops, kind, page):
    c = Case(ops, LENGTHS, kind, page=page, seed=page)
    c.check(attend(ops, c))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("D", [8, 16, 40, 64, 72, 80, 96, 128, 136, 192, 200, 256])
@pytest.mark.parametrize("page", [16, 20])
def test_head_sizes(ops, kind, D, page):
    c = Case(ops, [1, 45, 0, 200, 700], kind, Hq=6, Hkv=3, D=D, page=page, seed=D)
    c.check(attend(ops, c))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (16, 16), (7, 1), (15, 1), (16, 1), (17, 1), (32, 1), (33, 1), (64, 1), (130, 2), (48, 3), (40, 2)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_heads(ops, Hq, Hkv, D):
    c = Case(ops, [3, 400, 0, 77, 165], Hq=Hq, Hkv=Hkv, D=D, page=32, seed=Hq)
    c.check(attend(ops, c))


@pytest.mark.parametrize("page", [16, 7])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 33, 100, 128, 250, 516, 517, 10000])
def test_windows(ops, window, page):
    c = Case(ops, LENGTHS, "fp16", page=page, seed=window)
    c.check(attend(ops, c, window=window), window=window)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lengths", [[5000], [4096, 1, 2500], [9000, 0, 3, 3000, 129, 64, 1], [128] * 300, [20] * 70 + [3000] + [7] * 64])
def test_many_units(ops, kind, lengths):
    c = Case(ops, lengths, kind, Hq=4, Hkv=1, D=64, page=16, seed=len(lengths), spread=2.0)
    c.check(attend(ops, c))


def test_few_sequences_cut_finely(ops):
    # 256 workgroups' worth of heads, so that units are at their smallest and their largest
    for Hkv, n in ((2, 2000), (8, 1500), (64, 700)):
        c = Case(ops, [n, n // 3], Hq=Hkv, Hkv=Hkv, D=64, page=64, seed=Hkv)
        c.check(attend(ops, c))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 30.0])
def test_scales(ops, scale):
    # so far apart that one weight is all, or the same, or the other way round
    c = Case(ops, [1, 100, 600], seed=3)
    c.check(attend(ops, c, scale=scale), scale=scale)


@pytest.mark.parametrize("kind", TYPES)
def test_one_key_above_very_many(ops, kind):
    # weights of 2^-20 each that together count: small ones must not be lost
    n, D = 6000, 64
    c = Case(ops, [n], kind, Hq=2, Hkv=1, D=D, page=64, seed=8)
    k, q = torch.zeros_like(c.cache.k), torch.zeros_like(c.q)
    q[..., 0] = 1.0
    first = int(c.table[0, 0])
    k[first, 0, 0, 0] = 20 * np.log(2.0)
    c.cache.k.copy_(k)
    c.q.copy_(q)
    c.k64, c.q64 = k.double().cpu().numpy(), q.double().cpu().numpy()
    c.check(attend(ops, c, scale=1.0), scale=1.0)


@pytest.mark.parametrize("page", [16, 10])
def test_missing_pages(ops, page):
    c = Case(ops, [40, 200, 700, 33], page=page, seed=5)
    c.table[0] = -1                                   # none at all
    c.table[1, 2] = len(c.k64)                        # one past the last
    c.table[2, ::3] = np.iinfo(np.int32).min
    c.table[2, 10:30] = np.iinfo(np.int32).max
    c.table[3, 0] = -1                                # the first
    c.dtable.copy_(torch.from_numpy(c.table))
    got = attend(ops, c)
    c.check(got)
    assert not got[0][0].any() and torch.isinf(got[1][0]).all()


def test_cache_without_pages(ops):
    c = Case(ops, [3, 50])
    none = ops.PagedCache(c.cache.k[:0], c.cache.v[:0])
    out, lse = ops.cache_attention(c.q, none, c.dtable, c.dlengths, return_lse=True)
    assert not out.any() and (lse == float("-inf")).all()


def test_lengths_outside_the_table(ops):
    c = Case(ops, [48, 48, 48], page=16, seed=2)
    c.lengths[:] = [-7, 1 << 30, 48]
    c.dlengths.copy_(torch.from_numpy(c.lengths))
    assert c.table.shape[1] == 3
    c.check(attend(ops, c))


def test_no_columns_in_the_table_and_no_sequences(ops):
    c = Case(ops, [5, 6])
    out, lse = ops.cache_attention(c.q, c.cache, c.dtable[:, :0], c.dlengths, return_lse=True)
    assert not out.any() and (lse == float("-inf")).all()
    assert ops.cache_attention(c.q[:0], c.cache, c.dtable[:0], c.dlengths[:0]).shape == (0, 8, 128)


@pytest.mark.parametrize("page", [16, 9])
def test_infinities_and_nan(ops, page):
    # each stays with the heads and the columns that its formula gives it to
    c = Case(ops, [70, 70, 70, 300, 70], Hq=4, Hkv=2, D=64, page=page, seed=6)

    def put(which, b, j, h, d, x):
        p = int(c.table[b, j // page])
        (c.cache.k if which == "k" else c.cache.v)[p, h, j % page, d] = x
        (c.k64 if which == "k" else c.v64)[p, h, j % page, d] = x

    put("v", 0, 13, 0, 5, float("inf"))
    put("v", 1, 69, 1, 63, float("nan"))
    put("k", 2, 40, 0, 0, float("nan"))
    put("k", 3, 299, 1, 7, float("inf"))  # a head whose q is positive there: NaN; negative: that key has no weight
    put("v", 4, 0, 0, 0, float("-inf"))
    got = attend(ops, c)
    out, bound, lse, lse_bound = c.want()
    # weights are in two parts, of which one may be 0 or negative: infinite values give infinite results or NaN
    assert np.array_equal(np.isfinite(got[0].double().cpu().numpy()), np.isfinite(out))
    some = np.isfinite(out)
    near(torch.where(torch.from_numpy(some).cuda(), got[0], 0), np.where(some, out, 0), np.where(some, bound, 0))
    near(got[1], lse, lse_bound)


def test_scores_of_minus_infinity(ops):
    c = Case(ops, [50, 200], "bf16", Hq=2, Hkv=1, D=8, page=16, seed=7)
    c.q.fill_(1.0)
    c.q64[:] = 1.0
    for b, keep in ((0, []), (1, [150, 151])):
        for j in range(c.lengths[b]):
            if j not in keep:
                p = int(c.table[b, j // 16])
                c.cache.k[p, 0, j % 16, 3] = float("-inf")
                c.k64[p, 0, j % 16, 3] = -np.inf
    got = attend(ops, c)
    c.check(got)
    assert not got[0][0].any()


@pytest.mark.parametrize("kind", TYPES)
def test_strides(ops, kind):
    c = Case(ops, [200, 3, 700], kind, Hq=6, Hkv=2, D=72, page=12, seed=9, both=True, extra=3)
    want, lse = attend(ops, c)
    c.check((want, lse))
    # queries as a part of a projection's output, at an odd place; heads far apart; one for all sequences
    for pad in (8, 1):
        wide = torch.full((3, 6 * 72 + 2 * pad), float("nan"), dtype=c.q.dtype, device="cuda")
        q = wide[:, pad:pad + 6 * 72].unflatten(1, (6, 72))
        q.copy_(c.q)
        assert torch.equal(ops.cache_attention(q, c.cache, c.dtable, c.dlengths), want)
        wide = torch.full((3, 6, 72 + pad), float("nan"), dtype=c.q.dtype, device="cuda")
        wide[..., pad:] = c.q
        assert torch.equal(ops.cache_attention(wide[..., pad:], c.cache, c.dtable, c.dlengths), want)
        out = torch.full((3, 6 * 72 + pad), 7.0, dtype=c.q.dtype, device="cuda")
        view = out[:, pad:].unflatten(1, (6, 72))
        assert ops.cache_attention(c.q, c.cache, c.dtable, c.dlengths, out=view) is view
        assert torch.equal(view, want) and (out[:, :pad] == 7).all()
    q = c.q[:1].expand(3, -1, -1)
    assert torch.equal(ops.cache_attention(q, c.cache, c.dtable, c.dlengths), ops.cache_attention(q.contiguous(), c.cache, c.dtable, c.dlengths))
    t = c.dtable[2:].expand(3, -1)
    assert torch.equal(ops.cache_attention(q, c.cache, t, c.dlengths), ops.cache_attention(q, c.cache, t.contiguous(), c.dlengths))


def test_parts_join_by_the_logarithm(ops):
    # a sequence in two parts, by its pages, is what it is in one
    c = Case(ops, [640], "bf16", Hq=4, Hkv=2, D=64, page=64, seed=12)
    whole, lse = attend(ops, c)
    a, la = ops.cache_attention(c.q, c.cache, c.dtable[:, :3].contiguous(), c.dlengths, return_lse=True)
    b, lb = ops.cache_attention(c.q, c.cache, c.dtable[:, 3:].contiguous(), c.dlengths, return_lse=True)
    both = torch.logaddexp(la, lb)
    a, b = a.double() * torch.exp(la - both)[..., None].double(), b.double() * torch.exp(lb - both)[..., None].double()
    out, bound, lse64, lse_bound = c.want()
    # each part is rounded by itself, by up to half a step of what it adds; those add up where the parts cancel
    near(a + b, out, bound + ref.UNIT["bf16"] * (a.abs() + b.abs()).cpu().numpy())
    near(both, lse64, lse_bound)
    assert torch.allclose(both, lse, atol=1e-5)


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("T,Hkv,D,page", [(1, 1, 8, 1), (5, 3, 24, 7), (64, 8, 128, 16), (1000, 2, 72, 33), (300, 1, 256, 256)])
@pytest.mark.parametrize("how", ["plain", "fused", "odd", "expanded"])
def test_append(ops, kind, T, Hkv, D, page, how):
    g = torch.Generator().manual_seed(T)
    t = TYPES[kind]
    pages = -(-T // page) + 3
    k, v = (torch.randn(T, Hkv, D, generator=g).to(t) for _ in "kv")
    if how == "expanded":
        k = k[:1].expand(T, -1, -1)
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 2:
        slots[T // 2] = -1
        slots[T // 3] = pages * page
        slots[0] = 2 ** 62
    both = torch.randn(pages, 2, Hkv, page, D, generator=g).to(t).cuda()
    want = both.cpu().clone()
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            want[s // page, 0, :, s % page], want[s // page, 1, :, s % page] = k[i], v[i]
    if how == "fused":
        x = torch.cat((torch.zeros(T, 2, D, dtype=t), k, v), 1).cuda()
        dk, dv = x[:, 2:2 + Hkv], x[:, 2 + Hkv:]
    elif how == "odd":
        x = torch.zeros(T, Hkv, D + 3, dtype=t, device="cuda")
        x[..., 1:D + 1] = k.cuda()
        dk, dv = x[..., 1:D + 1], v.cuda()
    else:
        dk, dv = (k.cuda() if how == "plain" else k[:1].cuda().expand(T, -1, -1)), v.cuda()
    cache = ops.PagedCache(both[:, 0], both[:, 1])
    version = both._version
    assert ops.cache_append(cache, dk, dv, slots.cuda()) is None
    assert torch.equal(both.cpu(), want) and both._version > version
    ops.cache_append(cache, dk[:0], dv[:0], slots[:0].cuda())
    assert torch.equal(both.cpu(), want)


def test_append_then_attend_over_steps(ops):
    """Sequences that grow by a token a step, as a decode loop has them, on another stream and from a graph."""
    B, Hq, Hkv, D, page, steps = 3, 4, 2, 64, 8, 40
    g = torch.Generator().manual_seed(3)
    new = torch.randn(steps, 2, B, Hkv, D, generator=g).to(torch.bfloat16).cuda()
    q = torch.randn(steps, B, Hq, D, generator=g).to(torch.bfloat16).cuda()
    table = torch.randperm(B * 5, generator=g).reshape(B, 5).int().cuda()

    def decode(run):
        cache = ops.PagedCache(*(torch.full((B * 5, Hkv, page, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"))
        outs = []
        for s in range(steps):
            slots = (table[:, s // page].long() * page + s % page)
            outs.append(run(cache, new[s, 0], new[s, 1], slots, q[s], torch.full((B,), s + 1, dtype=torch.int32, device="cuda")).clone())
        return torch.stack(outs), cache

    def eager(cache, k, v, slots, q, lengths):
        ops.cache_append(cache, k, v, slots)
        return ops.cache_attention(q, cache, table, lengths)

    want, cache = decode(eager)
    k64, v64 = cache.k.double().cpu().numpy(), cache.v.double().cpu().numpy()
    out, bound, _, _ = ref.attention(q[-1].double().cpu().numpy(), k64, v64, table.cpu().numpy(), [steps] * B, "bf16")
    near(want[-1], out, bound)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = decode(eager)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)

    held = {}

    def replayed(cache, k, v, slots, q, lengths):
        if not held:
            held["in"] = [x.clone() for x in (k, v, slots, q, lengths)]
            held["cache"] = cache
            eager(cache, *held["in"])  # nothing is loaded for the first time in the capture
            torch.cuda.synchronize()
            held["graph"] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(held["graph"]):
                held["out"] = eager(cache, *held["in"])
        for x, y in zip(held["in"], (k, v, slots, q, lengths)):
            x.copy_(y)
        held["graph"].replay()
        other = eager(ops.PagedCache(cache.k.clone(), cache.v.clone()), k, v, slots, q, lengths)  # eager work between the replays
        torch.cuda.synchronize()
        assert torch.equal(held["out"], other)
        return held["out"]

    got, _ = decode(replayed)
    assert torch.equal(got, want)


def test_two_calls_at_once(ops):
    c = Case(ops, [900, 40, 2000], Hq=8, Hkv=1, D=64, seed=20)
    want = attend(ops, c)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for i in range(30):
        with torch.cuda.stream(streams[i % 3]):
            got.append(attend(ops, c))
    torch.cuda.synchronize()
    for o, l in got:
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])


# ------------------------------------------------------------------ refusals of the binding

def test_refusals(ops):
    from paper_2606_10440_amd import SimError
    c = Case(ops, [20, 30])
    k = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    good = dict(q=c.q, cache=c.cache, table=c.dtable, lengths=c.dlengths)
    P = ops.PagedCache
    for bad in [dict(q=c.q.float()), dict(q=c.q.half()), dict(q=c.q[0]), dict(q=c.q[:, :7]), dict(q=c.q[..., :64]), dict(q=c.q.cpu()),
                dict(q=c.q.transpose(1, 2)), dict(cache=(c.cache.k, c.cache.v)), dict(cache=P(c.cache.k, c.cache.v[:1])),
                dict(cache=P(c.cache.k.float(), c.cache.v.float())), dict(cache=P(c.cache.k[:, :, ::2], c.cache.v[:, :, ::2])),
                dict(cache=P(c.cache.k.transpose(1, 2), c.cache.v.transpose(1, 2))), dict(table=None),
                dict(table=c.dtable.long()), dict(table=c.dtable[:1]), dict(table=c.dtable[0]), dict(table=c.dtable.cpu()),
                dict(lengths=c.dlengths.long()), dict(lengths=c.dlengths[:1]), dict(window=-1), dict(scale=float("nan")),
                dict(out=torch.empty_like(c.q, dtype=torch.float32)), dict(out=c.q), dict(out=torch.empty_like(c.q)[:, :4]),
                dict(out=torch.empty_like(c.q).requires_grad_())]:
        with pytest.raises((SimError, TypeError)):
            ops.cache_attention(**{**good, **bad})
    for bad in [dict(k=k.half()), dict(k=k[:1]), dict(k=k[:, :1]), dict(v=k[..., :64]), dict(slots=slots.int()), dict(slots=slots[:1]),
                dict(slots=slots.cpu()), dict(k=k.cpu()), dict(cache=P(torch.zeros_like(c.cache.k).requires_grad_(), c.cache.v))]:
        with pytest.raises(SimError):
            ops.cache_append(**{**dict(cache=c.cache, k=k, v=k, slots=slots), **bad})


def test_results_in_memory_that_is_read_are_refused(ops):
    from paper_2606_10440_amd import SimError
    c = Case(ops, [20, 30])
    k = torch.zeros(2, *c.cache.k.shape[1::2], dtype=c.cache.k.dtype, device="cuda")
    for part in c.cache:
        with pytest.raises(SimError, match="share"):
            ops.cache_attention(c.q, c.cache, c.dtable, c.dlengths, out=part.reshape(-1)[:c.q.numel()].view_as(c.q))
    with pytest.raises(SimError, match="own"):
        ops.cache_append(ops.PagedCache(c.cache.k, c.cache.k), k, k, torch.zeros(2, dtype=torch.int64, device="cuda"))
