"""Attention over a paged cache from its definition in 64 bits (numpy), with a bound on what 32-bit arithmetic, weights in
two parts and one rounding to the output's type may add."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -23                      # one 32-bit rounding, also where it truncates
UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
PARTS = {"fp16": 2.0 ** -21, "bf16": 2.0 ** -16}  # a weight in two parts of the type
TINY = {"fp16": 2.0 ** -24, "bf16": 2.0 ** -133}


def attention(q, k, v, table, lengths, kind, scale=None, window=0):
    """q [B, Hq, D], k and v [pages, Hkv, page, D], all 64-bit: (out, bound, lse, bound of lse)."""
    B, Hq, D = q.shape
    pages, Hkv, page, _ = k.shape
    scale = D ** -0.5 if scale is None else scale
    out, bound = np.zeros((B, Hq, D)), np.zeros((B, Hq, D))
    lse, lse_bound = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    for b in range(B):
        n = min(max(int(lengths[b]), 0), table.shape[1] * page)
        j = np.arange(max(0, n - window) if window else 0, n)
        at = table[b][j // page] if len(j) else j
        j, at = j[(at >= 0) & (at < pages)], at[(at >= 0) & (at < pages)]
        if not len(j):
            continue
        for h in range(Hq):
            kk, vv = k[at, h // (Hq // Hkv), j % page], v[at, h // (Hq // Hkv), j % page]
            with np.errstate(invalid="ignore"):
                z = scale * (kk @ q[b, h])
                if (z == -np.inf).all():
                    continue
                top = z.max()
                p = np.where(z == -np.inf, 0.0, np.exp(z - top))
                total = p.sum()
                out[b, h] = p @ vv / total
                lse[b, h] = top + np.log(total)
                # a score: D products' sum, its scaling and the distance to the highest; e^x of that
                far = np.abs(scale) * (np.abs(kk) @ np.abs(q[b, h]))
                off = (D + 8) * U32 * (far.max() if np.isfinite(far).all() else 0.0) + 8 * U32 * np.abs(z - top)[p > 0].max(initial=0.0)
                # the same error in the sum of weights, sums of n terms, the cuts' and the waves' joints
                rel = 2 * off + PARTS[kind] + (len(j) + 64) * U32
                size = p @ np.abs(vv) / total
                most = np.abs(vv)[np.isfinite(vv)].max(initial=0.0)
                bound[b, h] = rel * size + UNIT[kind] * (np.abs(out[b, h]) + rel * size) + TINY[kind] + len(j) * 2.0 ** -38 * most
                lse_bound[b, h] = off + (len(j) + 64) * U32 + 4 * U32 * (np.abs(top) + np.log(total)) + 2.0 ** -22
    return out, bound, lse, lse_bound
