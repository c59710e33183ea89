"""Operators on the GPU against their 64-bit definitions (``ops_reference``):
sizes from nothing to several tiles, odd ones among them, strides, masks that
leave rows empty, infinities and NaN, other streams and graphs."""
from __future__ import annotations

import numpy as np
import pytest

from tests import ops_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_10440_amd import ops as o
    return o


def rand(seed, shape, kind, scale=1.0, pad=0):
    """A seeded tensor on the GPU, the left part of a wider buffer of NaN if pad, and its values in 64 bits."""
    g = np.random.default_rng(seed)
    v = torch.from_numpy(g.standard_normal(shape) * scale).to(TYPES[kind])
    if pad:
        wide = torch.full(shape[:-1] + (shape[-1] + pad,), float("nan"), dtype=TYPES[kind], device="cuda")
        wide[..., :shape[-1]] = v.cuda()
        return wide[..., :shape[-1]], v.double().numpy()
    return v.cuda(), v.double().numpy()


def back(t):
    return t.detach().double().cpu().numpy()


def check(got, want, bound):
    got = back(got)
    assert got.shape == want.shape
    off = np.abs(got - want)
    assert not np.isnan(got).any()
    assert (off <= bound).all(), (np.unravel_index(np.argmax(off - bound), off.shape), float((off - bound).max()))


# ------------------------------------------------------------------ 4 bits

SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (5, 256), (4, 257), (17, 600), (70, 1000), (257, 129), (33, 2048)]


def same_codes(q, x):
    codes, scales = ref.mx4_stored(x)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(q.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_quantize(ops, kind, shape, pad):
    x, v = rand(1, shape, kind, pad=pad)
    q = ops.mx4_quantize(x)
    same_codes(q, v)
    for out in TYPES:
        assert np.array_equal(back(ops.mx4_dequantize(q, TYPES[out])), ref.mx4_values(v))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("pad", [0, 2, 3])
def test_quantize_transposed(ops, kind, shape, pad):
    x, v = rand(2, shape, kind, pad=pad)
    q = ops.mx4_quantize(x, transpose=True)
    assert q.shape == shape[::-1]
    same_codes(q, v.T)


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_every_bf16(ops, transpose):
    # each finite bf16 value as the largest of a block and as an element under larger ones
    bits = np.arange(1 << 16, dtype=np.uint32) << 16
    v = bits.view(np.float32)
    v = v[np.isfinite(v)]
    rng = np.random.default_rng(3)
    x = np.zeros((len(v), 32), np.float32)
    x[:, 0] = v
    x[:, 1:] = v[:, None] * rng.uniform(-1, 1, (len(v), 31)).astype(np.float32)
    t = torch.from_numpy(x).to(torch.bfloat16)
    d = t.cuda().t().contiguous() if transpose else t.cuda()
    same_codes(ops.mx4_quantize(d, transpose=transpose), t.double().numpy())


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_every_fp16(ops, transpose):
    v = np.arange(1 << 16, dtype=np.uint16).view(np.float16)
    v = v[np.isfinite(v)]
    rng = np.random.default_rng(3)
    x = np.zeros((len(v), 32), np.float16)
    x[:, 0] = v
    x[:, 1:] = (v[:, None].astype(np.float32) * rng.uniform(-1, 1, (len(v), 31))).astype(np.float16)
    t = torch.from_numpy(x)
    d = t.cuda().t().contiguous() if transpose else t.cuda()
    same_codes(ops.mx4_quantize(d, transpose=transpose), x.astype(np.float64))


def test_rows_of_a_stored_tensor(ops):
    # any run of rows is a tensor of its own, its scales at a multiple of eight bytes
    x, v = rand(17, (7, 200), "bf16")
    w, vw = rand(18, (40, 200), "bf16")
    q, qw = ops.mx4_quantize(x), ops.mx4_quantize(w)
    part, pw = ops.Mx4(q.codes[1:4], q.scales[1:4], (3, 200)), ops.Mx4(qw.codes[3:38], qw.scales[3:38], (35, 200))
    assert torch.equal(ops.mx4_dequantize(part, torch.float32), ops.mx4_dequantize(q, torch.float32)[1:4])
    want = ops.mx4_matmul(q, qw, dtype=torch.float32)
    assert torch.equal(ops.mx4_matmul(part, pw, dtype=torch.float32), want[1:4, 3:38])


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_ties_and_extremes(ops, transpose):
    rows = []
    for e in (-149, -130, -128, -127, -126, -100, 0, 60, 125):
        scale = 2.0 ** e
        rows.append(np.array([7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 6.5] * 2) * scale)
        rows[-1][16:] *= -1
    x = np.array(rows).astype(np.float32)
    x[~np.isfinite(x)] = 0
    d = torch.from_numpy(x).cuda()
    d = d.t().contiguous() if transpose else d
    same_codes(ops.mx4_quantize(d, transpose=transpose), x.astype(np.float64))


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_blocks_with_nan_or_infinity(ops, transpose, bad):
    x = np.random.default_rng(4).standard_normal((3, 96)).astype(np.float32)
    x[1, 40] = bad
    d = torch.from_numpy(x).cuda()
    q = ops.mx4_quantize(d.t().contiguous() if transpose else d, transpose=transpose)
    same_codes(q, x.astype(np.float64))
    v = back(ops.mx4_dequantize(q, torch.float32))
    assert np.isnan(v[1, 32:64]).all() and np.isnan(v).sum() == 32


def test_leading_axes(ops):
    x, v = rand(5, (3, 4, 70), "bf16")
    q = ops.mx4_quantize(x)
    assert q.shape == (3, 4, 70)
    same_codes(q, v.reshape(12, 70))
    assert ops.mx4_dequantize(q, torch.float32).shape == (3, 4, 70)


# ------------------------------------------------------------------ products

PRODUCTS = [(1, 1, 1), (1, 300, 256), (2, 64, 512), (5, 17, 700), (16, 256, 1024), (17, 33, 31), (31, 95, 257), (33, 129, 300),
            (64, 64, 2048), (65, 200, 1000), (127, 130, 513), (128, 256, 256), (200, 260, 1300), (300, 513, 260), (257, 1000, 520),
            (512, 512, 768)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("mnk", PRODUCTS)
def test_product(ops, kind, mnk):
    M, N, K = mnk
    a, va = rand(6, (M, K), "bf16")
    b, vb = rand(7, (N, K), "bf16", scale=K ** -0.5)
    got = ops.mx4_matmul(ops.mx4_quantize(a), ops.mx4_quantize(b), dtype=TYPES[kind])
    check(got, *ref.product(ref.mx4_values(va), ref.mx4_values(vb), kind))


@pytest.mark.parametrize("kind", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("mnk", [(1, 96, 300), (1, 2048, 4096), (3, 100, 1000), (16, 70, 512), (40, 300, 257), (130, 140, 600)])
@pytest.mark.parametrize("pad", [0, 5])
def test_linear(ops, kind, mnk, pad):
    M, N, K = mnk
    x, vx = rand(8, (M, K), kind, pad=pad)
    w, vw = rand(9, (N, K), "bf16", scale=K ** -0.5)
    wide = torch.full((M, N + 3), 7.0, dtype=TYPES[kind], device="cuda")
    got = ops.mx4_matmul(x, ops.mx4_quantize(w), out=wide[:, :N])
    check(got, *ref.product(ref.mx4_values(vx), ref.mx4_values(vw), kind))
    assert (wide[:, N:] == 7.0).all()


def test_product_whole_numbers_exact(ops):
    # small whole numbers: every partial sum is exact, so the layout of every element and scale shows
    rng = np.random.default_rng(10)
    for M, N, K in [(33, 40, 300), (256, 256, 512), (130, 270, 1025), (3, 500, 777), (300, 300, 256)]:
        a = rng.choice([0, 1, 2, 3, 4, 6, -1, -2], (M, K)) * np.exp2(rng.integers(0, 4, (M, 1)))
        b = rng.choice([0, 1, 2, 3, -3, -4], (N, K)) * np.exp2(rng.integers(0, 3, (N, 1)))
        a[:, ::32], b[:, ::32] = 4, 4
        for j in range(0, K, 32):  # another scale for each block
            a[:, j:j + 32] *= 2.0 ** (j // 32 % 3)
            b[:, j:j + 32] *= 2.0 ** (j // 32 % 4)
        qa, qb = (ops.mx4_quantize(torch.from_numpy(v).float().cuda()) for v in (a, b))
        got = back(ops.mx4_matmul(qa, qb, dtype=torch.float32))
        assert np.array_equal(got, ref.mx4_values(a) @ ref.mx4_values(b).T), (M, N, K)


@pytest.mark.parametrize("mnk", [(2, 40, 300), (70, 80, 300), (300, 300, 512)])
def test_product_nan_stays_in_its_row_and_column(ops, mnk):
    M, N, K = mnk
    a, _ = rand(11, (M, K), "bf16")
    b, _ = rand(12, (N, K), "bf16")
    a[1, 5] = float("inf")
    b[7, 290] = float("nan")
    got = back(ops.mx4_matmul(ops.mx4_quantize(a), ops.mx4_quantize(b), dtype=torch.float32))
    bad = np.zeros((M, N), bool)
    bad[1], bad[:, 7] = True, True
    assert np.array_equal(np.isnan(got), bad)


@pytest.mark.parametrize("mnk", [(1, 64, 64), (70, 90, 130), (300, 257, 513)])
@pytest.mark.parametrize("kind", ["bf16", "fp16"])
def test_linear_gradient(ops, mnk, kind):
    M, N, K = mnk
    x, vx = rand(13, (M, K), kind)
    w, vw = rand(14, (N, K), kind, scale=K ** -0.5)
    dy, vdy = rand(15, (M, N), kind)
    dx, dw = ops.mx4_linear_grad(dy, x, w)
    held = ref.mx4_values
    check(dx, *ref.product(held(vdy), held(vw.T), kind))
    check(dw, *ref.product(held(vdy.T), held(vx.T), kind))
    x.requires_grad_(), w.requires_grad_()
    y = ops.mx4_linear(x, w)
    check(y, *ref.product(held(vx), held(vw), kind))
    y.backward(dy)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw)


def test_linear_gradient_one_of_two_and_strides(ops):
    M, N, K = 70, 90, 130
    x, vx = rand(13, (M, K), "bf16", pad=3)
    w, vw = rand(14, (N, K), "bf16", scale=K ** -0.5, pad=6)
    dy, vdy = rand(15, (M, N), "bf16", pad=1)
    both = ops.mx4_linear_grad(dy, x, w)
    check(both[0], *ref.product(ref.mx4_values(vdy), ref.mx4_values(vw.T), "bf16"))
    check(both[1], *ref.product(ref.mx4_values(vdy.T), ref.mx4_values(vx.T), "bf16"))
    dx, none = ops.mx4_linear_grad(dy, x, w, need=(True, False))
    assert none is None and torch.equal(dx, both[0])
    none, dw = ops.mx4_linear_grad(dy, x, w, need=(False, True))
    assert none is None and torch.equal(dw, both[1])
    e = torch.empty(0, N, dtype=torch.bfloat16, device="cuda")
    dx, dw = ops.mx4_linear_grad(e, torch.empty(0, K, dtype=torch.bfloat16, device="cuda"), w)
    assert dx.shape == (0, K) and (dw == 0).all() and dw.shape == (N, K)


def test_linear_gradient_against_differences(ops):
    # values that 4 bits hold exactly along either axis: then the layer is bilinear and differences are its gradient
    rng = np.random.default_rng(16)
    M, N, K = 32, 32, 64
    x, w, dy = (rng.choice([-2.0, -1.0, 1.0, 2.0, 4.0, 6.0], s) for s in ((M, K), (N, K), (M, N)))
    for m in (x, w, dy):
        m[0::32], m[:, 0::32] = 4.0, 4.0   # every block's scale is 1
    tx, tw, tdy = (torch.from_numpy(v).to(torch.bfloat16).cuda() for v in (x, w, dy))
    dx, dw = ops.mx4_linear_grad(tdy.float(), tx.float(), tw.float())
    loss = lambda a, b: float((dy * (a @ b.T)).sum())  # noqa: E731
    for i, j in [(0, 0), (5, 7), (31, 63)]:
        e = np.zeros((M, K))
        e[i, j] = 0.5
        assert back(dx)[i, j] == loss(x + e, w) - loss(x - e, w)
        e = np.zeros((N, K))
        e[i, j] = 0.5
        assert back(dw)[i, j] == loss(x, w + e) - loss(x, w - e)


# ------------------------------------------------------------------ router

def logits_of(seed, T, E, kind, pad=0):
    z, v = rand(seed, (T, E), kind, scale=1.5, pad=pad)
    return z, v


def masks(T, E, how, seed=20):
    rng = np.random.default_rng(seed)
    if how == "none":
        return None
    if how == "expert":
        m = rng.random(E) < 0.7
        m[rng.integers(E)] = True
        return m
    m = rng.random((T, E)) < 0.5
    m[::3] = False           # rows with nothing left
    if T > 1:
        m[1] = False
        m[1, E - 1] = True   # and one with a single expert
    return m


def check_route(r, want):
    e, w, off, order, rel = want
    assert np.array_equal(r.experts.cpu().numpy(), e)
    assert np.array_equal(r.offsets.cpu().numpy(), off)
    assert np.array_equal(r.order.cpu().numpy(), order)
    got = back(r.weights)
    assert np.array_equal(np.isnan(got), np.isnan(w))
    fine = ~np.isnan(w)
    assert (np.abs(got - w) <= rel * w + 2.0 ** -126)[fine].all()


ROUTES = [(1, 1, 1), (1, 8, 2), (3, 16, 16), (5, 17, 3), (8, 64, 6), (16, 33, 32), (63, 100, 4), (64, 128, 8), (65, 256, 8),
          (130, 40, 1), (200, 257, 5), (129, 1024, 10), (1000, 60, 4), (17, 300, 6), (64, 513, 32), (4096, 12, 2), (4097, 12, 2)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("tek", ROUTES)
@pytest.mark.parametrize("how", ["none", "expert", "token"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_and_gradient(ops, kind, tek, how, renorm):
    T, E, k = tek
    z, v = logits_of(21, T, E, kind, pad=3 if T % 2 else 0)
    m = masks(T, E, how)
    want = ref.route(v, k, m, renorm)
    dm = None if m is None else torch.from_numpy(m).cuda()
    if m is not None:  # what stands in masked places has no effect
        z = torch.where(dm, z, torch.tensor(float("nan"), dtype=z.dtype, device="cuda"))
    r = ops.moe_route(z, k, mask=dm, renormalize=renorm)
    check_route(r, want)
    g, vg = rand(22, (T, k), "fp32")
    g = torch.where(r.experts < 0, torch.tensor(float("nan"), device="cuda"), g)
    dz = ops.moe_route_grad(z, r.experts, g, mask=dm, renormalize=renorm)
    wz, bound = ref.route_grad(v, want[0], vg, m, renorm)
    check(dz, wz, bound + ref.UNIT[kind] * (np.abs(wz) + bound) + ref.TINY[kind])


@pytest.mark.parametrize("kind", TYPES)
def test_route_ties_and_lowest_values(ops, kind):
    low = float(torch.finfo(TYPES[kind]).min)
    v = np.array([[1, 1, 1, 1, 1, 1], [0.0, -0.0, 0.0, -0.0, -1, -1], [low] * 6, [low, -np.inf, 2, low, -np.inf, -np.inf],
                  [-np.inf] * 6, [3, 2, 3, 2, 3, 2]])
    z = torch.from_numpy(v).to(TYPES[kind]).cuda()
    for renorm in (True, False):
        check_route(ops.moe_route(z, 4, renormalize=renorm), ref.route(z.double().cpu().numpy(), 4, None, renorm))


def test_route_nan_and_infinity(ops):
    v = np.array([[1.0, np.nan, 2.0, 0.0], [0.0, np.inf, 1.0, 2.0], [5.0, 4.0, 3.0, 2.0]])
    r = ops.moe_route(torch.from_numpy(v).float().cuda(), 2)
    assert r.experts.cpu().tolist() == [[1, 2], [1, 3], [0, 1]]
    w = back(r.weights)
    assert np.isnan(w[0]).all() and np.isnan(w[1, 0]) and np.isfinite(w[2]).all()


def test_route_many_chunks(ops):
    # above 512 chunks of 64 tokens the counts are scanned by a kernel of their own
    for T, E, k in [(64 * 512, 24, 2), (64 * 512 + 1, 24, 2), (64 * 700 + 5, 130, 3)]:
        g = torch.Generator(device="cuda").manual_seed(T)
        z = torch.randn(T, E, generator=g, device="cuda")
        r = ops.moe_route(z, k)
        e = r.experts.cpu().numpy()
        top = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k].cpu().numpy()
        assert np.array_equal(e, top)
        flat = e.reshape(-1)
        assert np.array_equal(r.order.cpu().numpy(), np.argsort(flat, kind="stable"))
        assert np.array_equal(r.offsets.cpu().numpy(), np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E))]))


@pytest.mark.parametrize("renorm", [True, False])
def test_route_gradient_against_differences(ops, renorm):
    T, E, k = 6, 20, 4
    z, v = logits_of(23, T, E, "fp32")
    g, vg = rand(24, (T, k), "fp32")
    lz = z.clone().requires_grad_()
    r = ops.moe_route_train(lz, k, renormalize=renorm)
    (r.weights * g).sum().backward()
    h = 1e-5  # far below the gaps between the logits here; the third derivative adds h^2
    e0 = ref.route(v, k, None, renorm)[0]
    for t in range(T):
        for e in range(E):
            d = np.zeros((T, E))
            d[t, e] = h
            up, down = (ref.route(v + s * d, k, None, renorm) for s in (1, -1))
            assert np.array_equal(up[0], e0) and np.array_equal(down[0], e0)
            want = ((up[1] - down[1]) * vg).sum() / (2 * h)
            assert abs(float(lz.grad[t, e]) - want) < 2e-5 * (1 + np.abs(vg[t]).sum())


# ------------------------------------------------------------------ experts' layer

LAYERS = [(1, 4, 2, 64, 32), (1, 8, 8, 200, 70), (2, 5, 1, 33, 17), (7, 16, 3, 256, 128), (15, 3, 2, 130, 257), (16, 6, 4, 512, 96),
          (17, 40, 2, 128, 64), (33, 2, 2, 96, 48), (65, 12, 3, 160, 100), (130, 3, 2, 72, 40),
          # rows shorter than one load, ends of rows at every place in a load
          (1, 2, 1, 1, 1), (3, 4, 2, 7, 9), (40, 3, 2, 9, 5), (5, 4, 2, 8, 8), (6, 4, 2, 579, 323), (20, 4, 2, 453, 197),
          (90, 3, 2, 582, 199), (9, 5, 3, 1100, 716), (110, 2, 2, 77, 510),
          # many experts, many choices
          (5, 100, 4, 64, 32), (16, 256, 8, 64, 32), (3, 257, 2, 64, 32), (4, 40, 32, 64, 40)]


def layer_case(ops, seed, T, E, D, F, kind, weights, pad=0):
    x, vx = rand(seed, (T, D), kind, pad=pad)
    z, vz = logits_of(seed + 1, T, E, "fp32")
    w13, v13 = rand(seed + 2, (E, 2 * F, D), kind, scale=D ** -0.5)
    w2, v2 = rand(seed + 3, (E, D, F), kind, scale=F ** -0.5)
    if weights == "mx4":
        w13, w2 = ops.mx4_quantize(w13), ops.mx4_quantize(w2)
        v13 = ref.mx4_values(v13.reshape(-1, D)).reshape(E, 2 * F, D)
        v2 = ref.mx4_values(v2.reshape(-1, F)).reshape(E, D, F)
    return (x, z, w13, w2), (vx, vz, v13, v2)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("weights", ["same", "mx4"])
@pytest.mark.parametrize("case", LAYERS)
@pytest.mark.parametrize("how", ["none", "expert", "token"])
def test_layer(ops, kind, weights, case, how):
    T, E, k, D, F = case
    (x, z, w13, w2), (vx, vz, v13, v2) = layer_case(ops, 30, T, E, D, F, kind, weights, pad=1 if T % 2 else 0)
    m = masks(T, E, how, seed=T)
    dm = None if m is None else torch.from_numpy(m).cuda()
    wide = torch.full((T, D + 2), 7.0, dtype=x.dtype, device="cuda")
    got = ops.moe_layer(x, z, w13, w2, k, mask=dm, renormalize=T % 3 != 0, out=wide[:, :D])
    check(got, *ref.layer(vx, vz, v13, v2, k, m, T % 3 != 0, kind))
    assert (wide[:, D:] == 7.0).all()


@pytest.mark.parametrize("T,E,k", [(4, 6, 2), (40, 4, 2)])
@pytest.mark.parametrize("weights", ["same", "mx4"])
def test_layer_unused_experts_and_other_tokens_have_no_effect(ops, weights, T, E, k):
    (x, z, w13, w2), _ = layer_case(ops, 40, T, E, 64, 48, "bf16", weights)
    mask = torch.ones(E, dtype=torch.bool, device="cuda")
    mask[1] = False
    want = ops.moe_layer(x, z, w13, w2, k, mask=mask)
    if weights == "mx4":
        w13.scales[1 * 96:2 * 96] = 255
        w2.scales[1 * 64:2 * 64] = 255
    else:
        w13[1], w2[1] = float("nan"), float("inf")
    assert torch.equal(ops.moe_layer(x, z, w13, w2, k, mask=mask), want)
    x[2] = float("nan")
    got = ops.moe_layer(x, z, w13, w2, k, mask=mask)
    assert torch.isnan(got[2]).all()
    keep = torch.arange(T, device="cuda") != 2
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("T,E", [(1, 3), (5, 4), (16, 6), (40, 4)])
@pytest.mark.parametrize("kind,weights", [("bf16", "same"), ("fp16", "same"), ("bf16", "mx4")])
def test_layer_infinite_weights_reach_only_their_experts_tokens(ops, kind, weights, T, E):
    (x, z, w13, w2), _ = layer_case(ops, 43, T, E, 64, 48, kind, weights)
    at = torch.arange(T, device="cuda")
    z.zero_()
    z[at, (at + 1) % E], z[at, (at + 2) % E] = 2.0, 1.0  # all but expert 0 for the first, and so on
    want = ops.moe_layer(x, z, w13, w2, 2)
    hit = ((at + 1) % E == 0) | ((at + 2) % E == 0)
    if weights == "mx4":
        w2.scales[7, 0] = 255
    else:
        w2[0, 7, 3] = float("inf")
    got = ops.moe_layer(x, z, w13, w2, 2)
    assert not torch.isfinite(got[hit, 7]).any()
    want[hit, 7] = got[hit, 7] = 0
    assert torch.equal(got, want)


def test_layer_infinite_hidden_value(ops):
    # x large enough that silu(g) u passes the 32-bit range, to +inf: the result is the sign of each weight of w2 times inf
    for T in (3, 40):
        x = torch.full((T, 64), 2.0 ** 100, dtype=torch.bfloat16, device="cuda")
        w13 = torch.ones(1, 64, 64, dtype=torch.bfloat16, device="cuda")
        w2 = torch.ones(1, 64, 32, dtype=torch.bfloat16, device="cuda")
        w2[0, ::2] = -1
        got = ops.moe_layer(x, torch.zeros(T, 1, device="cuda"), w13, w2, 1)
        assert (got[:, ::2] == -float("inf")).all() and (got[:, 1::2] == float("inf")).all()


def test_layer_nan_scale_in_a_used_expert(ops):
    (x, z, w13, w2), _ = layer_case(ops, 41, 3, 2, 64, 64, "bf16", "mx4")
    w2.scales[5, 0] = 255   # row 5 of expert 0, every token takes both experts
    got = back(ops.moe_layer(x, z, w13, w2, 2))
    bad = np.zeros((3, 64), bool)
    bad[:, 5] = True
    assert np.array_equal(np.isnan(got), bad)


def test_layer_hidden_values_beyond_fp16(ops):
    # fp16 weights and inputs whose hidden values pass 65504 while the result does not
    T, E, k, D, F = 3, 2, 1, 64, 32
    (x, z, w13, w2), (vx, vz, v13, v2) = layer_case(ops, 42, T, E, D, F, "fp16", "same")
    w13 *= 400.0
    w2 *= 2.0 ** -10
    got = ops.moe_layer(x, z, w13, w2, k)
    check(got, *ref.layer(vx, vz, back(w13), back(w2), k, None, True, "fp16"))


def test_layer_repeats_bit_for_bit(ops):
    for T, E, k, D, F, weights in [(1, 8, 2, 512, 256, "same"), (16, 8, 2, 512, 256, "mx4"), (100, 8, 2, 512, 256, "same")]:
        (x, z, w13, w2), _ = layer_case(ops, 43, T, E, D, F, "bf16", weights)
        first = ops.moe_layer(x, z, w13, w2, k)
        for _ in range(5):
            assert torch.equal(ops.moe_layer(x, z, w13, w2, k), first)


# ------------------------------------------------------------------ empty, streams, graphs

def test_nothing_to_do(ops):
    z = torch.empty(0, 8, device="cuda")
    r = ops.moe_route(z, 2)
    assert r.experts.shape == (0, 2) and (r.offsets == 0).all() and r.offsets.numel() == 9 and r.order.numel() == 0
    assert ops.moe_route_grad(z, r.experts, torch.empty(0, 2, device="cuda")).shape == (0, 8)
    assert ops.mx4_quantize(torch.empty(2, 3, 0, device="cuda")).codes.shape == (6, 0)
    q = ops.mx4_quantize(torch.empty(0, 64, device="cuda"))
    assert ops.mx4_dequantize(q).shape == (0, 64)
    w = ops.mx4_quantize(torch.randn(5, 64, device="cuda"))
    assert ops.mx4_matmul(q, w).shape == (0, 5)
    e0 = ops.mx4_quantize(torch.empty(3, 0, device="cuda"))
    assert (ops.mx4_matmul(e0, ops.mx4_quantize(torch.empty(4, 0, device="cuda"))) == 0).all()
    x = torch.empty(0, 32, dtype=torch.bfloat16, device="cuda")
    w13, w2 = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((8, 16, 32), (8, 32, 8)))
    assert ops.moe_layer(x, z, w13, w2, 2).shape == (0, 32)
    y = ops.moe_layer(torch.ones(3, 32, dtype=torch.bfloat16, device="cuda"), torch.randn(3, 8, device="cuda"),
                      w13[:, :0], w2[:, :, :0].contiguous(), 2)
    assert (y == 0).all()


def step(ops, x, z, w13, w2, wq, g):
    r = ops.moe_route(z, 2)
    return (ops.moe_layer(x, z, w13, w2, 2), r.experts, r.weights, r.offsets, r.order,
            ops.moe_route_grad(z, r.experts, g), ops.mx4_matmul(x, wq), ops.mx4_dequantize(ops.mx4_quantize(x, transpose=True)))


@pytest.mark.parametrize("T", [2, 100])
def test_other_stream_and_graph(ops, T):
    (x, z, w13, w2), _ = layer_case(ops, 50, T, 8, 256, 64, "bf16", "same")
    wq = ops.mx4_quantize(torch.randn(300, 256, device="cuda"))
    g = torch.randn(T, 2, device="cuda")
    args = (x, z, w13, w2, wq, g)
    want = [t.clone() for t in step(ops, *args)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(ops, *args)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step(ops, *args)
    for i in range(4):
        x2, z2 = torch.randn_like(x), torch.randn_like(z)
        x.copy_(x2), z.copy_(z2)
        graph.replay()
        torch.cuda.synchronize()
        eager = step(ops, *args)
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), i


def test_binding_refuses_tensors_that_do_not_fit(ops):
    from paper_2606_10440_amd.sim import SimError
    x = torch.randn(4, 64, device="cuda").bfloat16()
    w, z = ops.mx4_quantize(torch.randn(8, 64, device="cuda")), torch.randn(4, 8, device="cuda")
    r = ops.moe_route(z, 2)
    dw, mask = torch.ones(4, 2, device="cuda"), torch.ones(4, 8, dtype=torch.bool, device="cuda")
    w13, w2 = torch.zeros(8, 32, 64, device="cuda").bfloat16(), torch.zeros(8, 64, 16, device="cuda").bfloat16()
    Mx4 = ops.Mx4
    for i, call in enumerate([
            lambda: ops.mx4_quantize(x.double()), lambda: ops.mx4_quantize(x[:, ::2]), lambda: ops.mx4_quantize(x.cpu()),
            lambda: ops.mx4_quantize(x[:1].expand(4, 64)), lambda: ops.mx4_quantize(x[0, 0]), lambda: ops.mx4_quantize(None),
            lambda: ops.mx4_quantize(x[0], transpose=True),
            lambda: ops.mx4_dequantize(x), lambda: ops.mx4_dequantize(w, torch.float64), lambda: ops.mx4_dequantize(w, "bf16"),
            lambda: ops.mx4_dequantize(Mx4(w.codes[:, :64], w.scales, w.shape)),
            lambda: ops.mx4_dequantize(Mx4(w.codes, w.scales, (8, 300))),
            lambda: ops.mx4_dequantize(Mx4(w.codes, w.scales, (-8, 64))),
            lambda: ops.mx4_dequantize(Mx4(w.codes, w.scales, (1 << 39, 1 << 39, 64))),
            lambda: ops.mx4_dequantize(Mx4(w.codes, w.scales, ())), lambda: ops.mx4_dequantize(Mx4(w.codes, w.scales, 8)),
            lambda: ops.mx4_dequantize(Mx4(w.codes, w.scales.cpu(), w.shape)),
            lambda: ops.mx4_dequantize(Mx4(w.codes.view(torch.int8), w.scales, w.shape)),
            lambda: ops.mx4_matmul(x[:, :32], w), lambda: ops.mx4_matmul(x, x), lambda: ops.mx4_matmul(x, w, dtype=torch.int32),
            lambda: ops.mx4_matmul(x, Mx4(w.codes, w.scales, (2, 4, 64))),
            lambda: ops.mx4_matmul(Mx4(w.codes, w.scales, (2, 4, 64)), w),
            lambda: ops.mx4_matmul(x, w, out=torch.empty(4, 9, device="cuda")),
            lambda: ops.mx4_matmul(w, w, out=torch.empty(8, 8)), lambda: ops.mx4_matmul(x, w, out=z.to(torch.int32)),
            lambda: ops.mx4_linear_grad(z, x, w2[:, :, 0]), lambda: ops.mx4_linear_grad(z.bfloat16(), x, torch.zeros(8, 64, device="cuda")),
            lambda: ops.moe_route(z, 0), lambda: ops.moe_route(z, 9), lambda: ops.moe_route(z, 2, mask=mask.float()),
            lambda: ops.moe_route(z, 2, mask=mask[0, :7]), lambda: ops.moe_route(z, 2, mask=mask.cpu()),
            lambda: ops.moe_route(z, 2, mask=mask.t().contiguous().t()), lambda: ops.moe_route(z, 2, mask=mask[:3]),
            lambda: ops.moe_route(torch.zeros(2, 1025, device="cuda"), 2),
            lambda: ops.moe_route_grad(z, r.experts.long(), dw), lambda: ops.moe_route_grad(z, r.experts, dw.half()),
            lambda: ops.moe_route_grad(z, r.experts[:3], dw[:3]), lambda: ops.moe_route_grad(z, r.experts, dw.t().contiguous().t()),
            lambda: ops.moe_route_grad(z, r.order, dw), lambda: ops.moe_route_grad(z, r.experts, dw.cpu()),
            lambda: ops.moe_layer(x.float(), z, w13, w2, 2), lambda: ops.moe_layer(x[:3], z, w13, w2, 2),
            lambda: ops.moe_layer(x, z, w13.half(), w2, 2), lambda: ops.moe_layer(x, z, w13, w, 2),
            lambda: ops.moe_layer(x, z, w13[:, :30].contiguous(), w2, 2), lambda: ops.moe_layer(x, z, w13[:, :, ::2], w2, 2),
            lambda: ops.moe_layer(x, z[:, :7].contiguous(), w13, w2, 2), lambda: ops.moe_layer(x, z, w13.cpu(), w2, 2),
            lambda: ops.moe_layer(x, z, w13, w2, 2, out=torch.empty(4, 64, device="cuda")),
            lambda: ops.moe_layer(x, z, w13, w2, 2, out=x[:, :63])]):
        with pytest.raises(SimError):
            call()
            print("not refused:", i)
    with pytest.raises(TypeError):
        ops.moe_route(z, "2")
    assert torch.equal(ops.mx4_dequantize(Mx4(w.codes, w.scales, torch.Size((2, 4, 64)))).view(8, 64), ops.mx4_dequantize(w))


@pytest.mark.parametrize("shape", [(2, 3, 70), (5,), (2, 2, 2, 300), (0, 4, 64)])
def test_shapes_of_any_rank(ops, shape):
    x = torch.randn(shape, device="cuda")
    q = ops.mx4_quantize(x)
    flat = ops.mx4_quantize(x.reshape(-1, shape[-1]) if x.numel() else x.new_empty(0, shape[-1]))
    assert type(q) is ops.Mx4 and type(q.shape) is tuple and q.shape == shape
    assert torch.equal(q.codes, flat.codes) and torch.equal(q.scales, flat.scales)
    assert ops.mx4_dequantize(q).shape == shape
