"""The router with scores, bias and groups from its definition in 64 bits (numpy), and its gradient."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -23


def allowed(z, mask):
    ok = np.ones(z.shape, bool) if mask is None else np.broadcast_to(np.asarray(mask, bool), z.shape)
    return ok & ~(z == -np.inf)


def scores(z, ok, score):
    """64-bit scores, 0 where not allowed."""
    with np.errstate(over="ignore", invalid="ignore"):
        if score == "sigmoid":
            e = np.exp(-np.abs(z))
            s = np.where(z < 0, e, 1.0) / (1.0 + e)
        else:
            top = np.where(ok, z, -np.inf).max(1, keepdims=True)
            top = np.where(np.isnan(np.where(ok, z, 0.0)).any(1, keepdims=True), np.nan, top)
            p = np.where(ok, np.exp(np.where(ok, z - top, 0.0)), 0.0)
            total = p.sum(1, keepdims=True)
            s = np.divide(p, total, out=np.zeros_like(p), where=~(total == 0))
    return np.where(ok, s, 0.0)


def falling(values):
    """Sort key of a value: NaN above every number, then falling."""
    return (0, 0.0) if np.isnan(values) else (1, -float(values))


def route(z, k, mask=None, renorm=True, score="softmax", bias=None, groups=1, top_groups=None, best=1, scale=1.0):
    """(experts, weights, offsets, order)"""
    T, E = z.shape
    top_groups = groups if top_groups is None else top_groups
    size = E // groups
    ok = allowed(z, mask)
    s = scores(z, ok, score)
    with np.errstate(invalid="ignore", over="ignore"):
        c = s.astype(np.float32) + (np.float32(0) if bias is None else np.asarray(bias, np.float32))
    by = z if bias is None else c
    experts, weights = np.full((T, k), -1, np.int64), np.zeros((T, k))
    for t in range(T):
        can = [e for e in range(E) if ok[t, e] and not (bias is not None and c[t, e] == -np.inf)]
        if top_groups < groups:
            value = {}
            for g in range(groups):
                of = [e for e in can if e // size == g]
                if not of:
                    continue
                if best == 1:
                    value[g] = min(falling(by[t, e]) for e in of)
                else:
                    two = sorted((c[t, e] for e in of), key=falling)[:2]
                    with np.errstate(invalid="ignore", over="ignore"):
                        value[g] = falling(two[0] + two[1] if len(two) == 2 else two[0])
            keep = sorted(value, key=lambda g: (value[g], g))[:top_groups]
            can = [e for e in can if e // size in keep]
        pick = sorted(can, key=lambda e: (falling(by[t, e]), e))[:k]
        if not pick:
            continue
        experts[t, :len(pick)] = pick
        w = s[t, pick]
        if renorm:
            with np.errstate(invalid="ignore"):
                if score == "sigmoid":  # so far down that 64 bits do not hold the scores
                    x = z[t, pick]
                    w = np.exp(np.minimum(x, 0) - min(0, x.max())) / (1 + np.exp(-np.abs(x)))
                else:
                    w = np.exp(z[t, pick] - z[t, pick].max())
                    if np.isnan(s[t, pick]).any():
                        w = w * np.nan if np.isnan(z[t, pick]).any() else w
                w = w / w.sum()
        weights[t, :len(pick)] = w * scale
    flat = experts.reshape(-1)
    valid = np.nonzero(flat >= 0)[0]
    order = np.full(T * k, -1, np.int64)
    order[:len(valid)] = valid[np.argsort(flat[valid], kind="stable")]
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[valid], minlength=E))])
    return experts, weights, offsets, order


def grad(z, experts, g, mask=None, renorm=True, score="softmax", scale=1.0):
    """(d_logits, bound of 32-bit arithmetic): 32-bit exponentials of arguments up to 104, sums of E / 16 + 32 terms, eight products."""
    T, E = z.shape
    ok = allowed(z, mask)
    s = scores(z, ok, score)
    dz, bound = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        at = [j for j in range(experts.shape[1]) if experts[t, j] >= 0 and ok[t, experts[t, j]]]
        if not at:
            continue
        sel = experts[t, at]
        gs = g[t, at] * scale
        x = z[t, sel]
        p = s[t, sel]
        if renorm:
            p = np.exp(np.minimum(x, 0) - min(0, x.max())) / (1 + np.exp(-np.abs(x))) if score == "sigmoid" else np.exp(x - x.max())
            p = p / p.sum()
        far = min(104.0, np.abs(z[t][ok[t]]).max() * 2)
        rel = 3 * (E / 16 + 32 + far) * U32
        dot = (gs * p).sum() if renorm or score == "softmax" else 0.0
        size = (np.abs(gs) * p).sum() if renorm or score == "softmax" else 0.0
        rest = 1 / (1 + np.exp(np.clip(x, -700, 700))) if score == "sigmoid" else 1.0
        if renorm or score == "sigmoid":
            dz[t, sel] = p * (gs - dot) * rest
            bound[t, sel] = rel * p * (np.abs(gs) + size) * rest
        else:
            dz[t] = -s[t] * dot
            dz[t, sel] += p * gs
            bound[t] = rel * s[t] * size
            bound[t, sel] += rel * p * np.abs(gs)
    return dz, bound
