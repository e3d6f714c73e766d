"""Token sampling with temperature, top-k, top-p and min-p (taps_sample): one row at a time,
the whole vocabulary sorted, integer weights in Python's exact arithmetic."""
from __future__ import annotations

import math

import numpy as np

ONE = 1 << 43


def weights(v: np.ndarray, T: float) -> np.ndarray:
    """Integer weights of values in rank order (largest first, NaN last)."""
    with np.errstate(invalid="ignore", over="ignore"):
        t = (v - v[0]) / T
        w = np.rint(np.exp(np.where(np.isnan(t), -np.inf, t)) * ONE).astype(np.int64)
    w[v == v[0]] = ONE
    w[np.isnan(v)] = 0
    return w


def sample_row(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Returns (token, probability) of one row of logits (any float type, exact in fp64); the
    settings are taken as the values given."""
    x = np.asarray(x, np.float64)
    V = len(x)
    order = np.lexsort((np.arange(V), np.where(np.isnan(x), np.inf, -x), np.isnan(x)))
    v = x[order]
    if np.isnan(v[0]):
        return 0, 0.0
    if not temperature > 0:
        return int(order[0]), 1.0
    w = weights(v, temperature)
    cum = np.cumsum(w)                      # below 2^63: at most 2^20 weights of 2^43
    n = top_k if 0 < top_k < V else V
    if top_p < 1:
        need = max(1, math.ceil(max(top_p, 0.0) * int(cum[n - 1])))
        n = min(n, int(np.searchsorted(cum, need, side="left")) + 1)
    if min_p > 0:
        with np.errstate(invalid="ignore"):
            keep = (v == v[0]) | ((v - v[0]) / temperature >= min(math.log(min_p), 0.0))
        n = min(n, int(keep.sum()))
    S = int(cum[n - 1])
    u = min(max(u, 0.0), 1.0) if u == u else 0.0
    target = min(math.floor(u * S), S - 1)
    r = int(np.searchsorted(cum, target, side="right"))
    return int(order[r]), int(w[r]) / S


def sample(logits, u, n_nodes=None, temperature=None, top_k=None, top_p=None, min_p=None):
    """logits [B][N][V]; returns tokens and probabilities [B][N] (-1 and 0 past n_nodes)."""
    B, N, _ = logits.shape
    tok, pr = np.full((B, N), -1, np.int32), np.zeros((B, N))
    for b in range(B):
        kw = {}
        if temperature is not None:
            kw["temperature"] = float(temperature[b])
        if top_k is not None:
            kw["top_k"] = int(top_k[b])
        if top_p is not None:
            p = float(top_p[b])
            kw["top_p"] = 1.0 if math.isnan(p) else p
        if min_p is not None:
            kw["min_p"] = float(min_p[b])
        for i in range(N if n_nodes is None else min(max(int(n_nodes[b]), 0), N)):
            tok[b, i], pr[b, i] = sample_row(logits[b, i], float(u[b, i]), **kw)
    return tok, pr
