"""Traffic of an expert-parallel step: which 128 B lines a router's choices
put on the network.

Tokens and experts are spread over the endpoints in blocks.  A token goes
once to every other endpoint that has one of its experts (dispatch), and
every such endpoint sends one partial result back (combine).  What stays on
its endpoint is no traffic.  This module only lists transfers; it performs
none of the simulated method's arithmetic.
"""
from __future__ import annotations

import numpy as np

from . import LINE_BYTES


def lines_of(n_bytes: int) -> int:
    """Whole lines that n_bytes take."""
    return -(-n_bytes // LINE_BYTES)


def lines_of_token(q) -> int:
    """Lines that one row of a 4-bit tensor (``ops.Mx4``) takes: its codes,
    then its scales, as they are stored."""
    return lines_of(q.codes.shape[1]) + lines_of(q.scales.shape[1])


def token_moves(experts, n_experts: int, n_ranks: int):
    """(home, away) endpoint pairs, one for each token and each other endpoint
    that has one of its experts; in token order.  ``experts`` is [T, k], -1
    where a token has fewer."""
    experts = np.asarray(experts)
    T = len(experts)
    home = np.arange(T, dtype=np.int64) * n_ranks // max(T, 1)
    owner = experts.astype(np.int64) * n_ranks // n_experts
    goes = np.zeros((T, n_ranks), bool)
    t, j = np.nonzero(experts >= 0)
    goes[t, owner[t, j]] = True
    goes[np.arange(T), home] = False
    t, away = np.nonzero(goes)
    return home[t].astype(np.int32), away.astype(np.int32)


def transfers(src, dst, lines_each: int):
    """Source and destination of every line where each move takes so many."""
    return np.repeat(np.asarray(src, np.int32), lines_each), np.repeat(np.asarray(dst, np.int32), lines_each)
