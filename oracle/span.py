"""Attention of rows over a window of their sequence's tokens and its first ones, in 64 bits, from the definition."""
from __future__ import annotations

import numpy as np


def attend(q, k, v, first, scale, window=1 << 40, sinks=0, rows=None):
    """q float64 [n][Hq][D] at positions first, first + 1, ..; k, v float64 [tokens][Hkv][D].  Row at p: tokens j <= p with p - j < window or j < sinks.
    Returns the outputs, and sum p_j |v_j| / sum p_j, for all rows or those whose indexes are given.  Tokens that a row does not attend over have no part in it."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    rows = range(n) if rows is None else rows
    out, size = np.zeros((len(rows), Hq, D)), np.zeros((len(rows), Hq, D))
    for i, t in enumerate(rows):
        p = first + t
        at = np.arange(max(0, p - window + 1), p + 1)
        at = np.concatenate([np.arange(min(sinks, int(at[0]))), at])
        kk, vv = k[at], v[at]
        x = np.einsum("hgd,jhd->hgj", q[t].reshape(-1, G, D), kk) * scale
        with np.errstate(invalid="ignore"):
            x = np.exp(x - x.max(-1, keepdims=True))
            x /= x.sum(-1, keepdims=True)
            out[i] = np.einsum("hgj,jhd->hgd", x, vv).reshape(Hq, D)
            size[i] = np.einsum("hgj,jhd->hgd", x, np.abs(vv)).reshape(Hq, D)
    return out, size
