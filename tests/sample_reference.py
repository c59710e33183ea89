"""Sampling from its definition in 64 bits (numpy), one row at a time."""
from __future__ import annotations

import numpy as np


def kept(z, temperature, top_k, top_p, min_p):
    """(indices that are kept, in the logits' falling order, their weights); None where the row has no finite highest logit."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or not np.isfinite(z.max()):
        return None
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    if not temperature > 0:
        return order[:1], np.ones(1)
    with np.errstate(over="ignore"):
        w = np.exp((z[order] - z[order[0]]) * (1.0 / np.float64(temperature)))
    n = top_k if 0 < top_k < len(z) else len(z)
    order, w = order[:n], w[:n]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int((before < np.float64(top_p) * w.sum()).sum()))
        order, w = order[:n], w[:n]
    if min_p > 0:
        n = max(1, int((w >= np.float64(min_p)).sum()))
        order, w = order[:n], w[:n]
    return order, w


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    k = kept(z, np.float32(temperature), int(top_k), np.float32(top_p), np.float32(min_p))
    if k is None:
        return -1
    u = np.float64(np.float32(u)) if u > 0 else 0.0
    u = min(u, 1 - 2.0 ** -24)
    place = np.argsort(k[0])
    order, w = k[0][place], k[1][place]
    order, w = order[w > 0], w[w > 0]
    cum = np.cumsum(w)
    return int(order[min(len(order) - 1, int((cum <= u * cum[-1]).sum()))])
