"""The operators from their definitions in 64 bits (numpy), with bounds on
what 32-bit sums and one rounding to the output's type may add."""
from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
U32 = 2.0 ** -23                       # one 32-bit rounding, also where it truncates
UNIT = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}  # rounding to the type, relative
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -24, "bf16": 2.0 ** -133}


def mx4_parts(x):
    """(codes [R, K32] 0..15, scale bytes [R, K32 / 32]) of x [R, K], K padded to whole blocks."""
    x = np.asarray(x, np.float64)
    R, K = x.shape
    full = np.zeros((R, -(-K // 32) * 32))
    full[:, :K] = x
    b = full.reshape(R, -1, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(b).max(2)
    bad = ~np.isfinite(top)
    _, e = np.frexp(np.where(bad | (top == 0), 1.0, top))   # top = m 2^e, m in [0.5, 1)
    s = np.where(top == 0, -127, np.maximum(e - 3, -127))
    a = np.abs(np.where(bad[:, :, None], 0.0, b)) / np.exp2(s.astype(np.float64))[:, :, None]
    code = np.zeros(a.shape, np.int64)
    for i in range(7):
        half = (GRID[i] + GRID[i + 1]) / 2
        code = np.where((a >= half) if i % 2 else (a > half), i + 1, code)
    code |= np.where(np.signbit(b) & ~bad[:, :, None], 8, 0)
    return code.reshape(R, -1), np.where(bad, 255, s + 127)


def mx4_stored(x):
    """Codes and scales in the stored layout."""
    code, byte = mx4_parts(x)
    R, K = np.asarray(x).shape
    g = -(-K // 256)
    c = np.zeros((R, g * 256), np.uint8)
    c[:, :code.shape[1]] = code
    s = np.zeros((R, g * 8), np.uint8)
    s[:, :byte.shape[1]] = byte
    return c[:, 0::2] | (c[:, 1::2] << 4), s


def mx4_values(x):
    code, byte = mx4_parts(x)
    v = np.where(code & 8, -1.0, 1.0) * GRID[code & 7]
    scale = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (v.reshape(len(v), -1, 32) * scale[:, :, None]).reshape(len(v), -1)[:, :np.asarray(x).shape[1]]


def product(a, b, kind):
    """a @ b.T and how far a kernel's result may be from it: every 32-bit sum of K products, in any order."""
    want = a @ b.T
    bound = (a.shape[1] + 1) * U32 * (np.abs(a) @ np.abs(b).T)
    return want, bound + UNIT[kind] * (np.abs(want) + bound) + TINY[kind]


def route(z, k, mask, renorm):
    """(experts, weights, offsets, order, relative bound on the weights)."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    ok = np.ones((T, E), bool) if mask is None else np.broadcast_to(np.asarray(mask, bool), (T, E))
    experts = np.full((T, k), -1, np.int64)
    weights = np.zeros((T, k))
    far = np.zeros((T, 1))
    for t in range(T):
        cand = [e for e in range(E) if ok[t, e] and not z[t, e] == -np.inf]
        cand.sort(key=lambda e: (0, 0.0, e) if np.isnan(z[t, e]) else (1, -z[t, e], e))
        pick = cand[:k]
        if not pick:
            continue
        with np.errstate(invalid="ignore"):
            p = np.exp(z[t, cand] - (np.nan if np.isnan(z[t, cand]).any() else z[t, cand].max()))
        experts[t, :len(pick)] = pick
        w = p[:len(pick)] / p.sum()
        weights[t, :len(pick)] = w / w.sum() if renorm else w
        fin = z[t, cand][np.isfinite(z[t, cand])]
        far[t] = min(104.0, fin.max() - fin.min()) if len(fin) else 0.0
    flat = experts.reshape(-1)
    valid = np.nonzero(flat >= 0)[0]
    order = valid[np.argsort(flat[valid], kind="stable")]
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[valid], minlength=E))])
    order = np.concatenate([order, np.full(T * k - len(valid), -1, np.int64)])
    # exp (2 roundings and its argument's own), the sums over 16 lanes, one division
    return experts, weights, offsets, order, (E / 16 + 16 + far) * U32


def route_grad(z, experts, g, mask, renorm):
    """(d_logits, absolute bound of 32-bit arithmetic)."""
    z = np.asarray(z, np.float64)
    T, E = z.shape
    ok = np.ones((T, E), bool) if mask is None else np.broadcast_to(np.asarray(mask, bool), (T, E))
    dz, bound = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        pick = [(j, e) for j, e in enumerate(experts[t]) if e >= 0]
        if not pick:
            continue
        sel = np.array([e for _, e in pick])
        gs = np.zeros(E)
        gs[sel] = [g[t, j] for j, _ in pick]
        use = np.zeros(E, bool)
        use[sel if renorm else np.nonzero(ok[t])[0]] = True
        v = np.where(use, z[t], -np.inf)
        p = np.exp(v - v.max())
        p /= p.sum()
        dz[t] = p * (gs - (gs * p).sum())
        fin = v[np.isfinite(v)]
        rel = (E / 16 + 16 + min(104.0, fin.max() - fin.min())) * U32
        bound[t] = 3 * rel * p * (np.abs(gs) + (np.abs(gs) * p).sum())
    return dz, bound


def layer(x, z, w13, w2, k, mask, renorm, kind):
    """(y, bound) of the experts' layer; 16 bits kept of the hidden values."""
    T, D = x.shape
    E, _, F = w2.shape
    experts, weights, _, _, rel = route(z, k, mask, renorm)
    rel = np.broadcast_to(rel, (T, 1))
    y, err = np.zeros((T, D)), np.zeros((T, D))
    for t in range(T):
        for j in range(k):
            e = experts[t, j]
            if e < 0:
                continue
            gu, size = w13[e] @ x[t], np.abs(w13[e]) @ np.abs(x[t])
            dgu = (D + 8) * U32 * size
            with np.errstate(over="ignore"):
                sg = gu[:F] / (1 + np.exp(-gu[:F]))
            h = sg * gu[F:] * weights[t, j]
            dh = weights[t, j] * (1.1 * dgu[:F] * np.abs(gu[F:]) + np.abs(sg) * dgu[F:] + 1.1 * dgu[:F] * dgu[F:])
            dh += np.abs(h) * (2.0 ** -16 + 16 * U32 + rel[t]) + np.abs(weights[t, j] * gu[F:]) * 2.0 ** -120
            y[t] += w2[e] @ h
            err[t] += np.abs(w2[e]) @ dh + (F + k + 8) * U32 * (np.abs(w2[e]) @ np.abs(h))
    return y, err + UNIT[kind] * (np.abs(y) + err) + TINY[kind]
