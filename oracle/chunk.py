"""Attention of chunks of new tokens over a paged cache (chunk_attn_paged), fp64."""
from __future__ import annotations

import numpy as np


def chunk_attention_paged(Q, K_pages, V_pages, table, q_start, kv_len, scale, window=0):
    """Q [rows][Hq][hd]; returns O (NaN in rows of no request) and, for error bounds, the sums of
    the weighted |v| per output, the largest sum_d |q_d k_d| per row and head, and the number of
    keys per row."""
    rows, Hq, hd = Q.shape
    pr, Hkv = K_pages.shape[1], K_pages.shape[2]
    G = Hq // Hkv
    O, A = np.full(Q.shape, np.nan), np.zeros(Q.shape)
    D, N = np.zeros((rows, Hq)), np.zeros(rows, dtype=np.int64)
    for b in range(len(kv_len)):
        first, end, kv = int(q_start[b]), int(q_start[b + 1]), int(kv_len[b])
        n = end - first
        if n <= 0:
            continue
        O[first:end] = 0.0
        at = kv - n + np.arange(n)                       # the tokens' rows
        low = max(0, int(at[0]) - window + 1) if window else 0
        if kv <= low:
            continue
        r = np.arange(low, kv)
        pages, slot = table[b, r // pr], r % pr
        gap = at[:, None] - r[None, :]
        seen = (gap >= 0) & (gap < window) if window else gap >= 0
        N[first:end] = seen.sum(1)
        live = seen.any(1)
        if not live.any():
            continue
        sl = np.arange(first, end)[live]
        seen = seen[live]
        for g in range(Hkv):
            k = K_pages[pages, slot, g].astype(np.float64)
            v = V_pages[pages, slot, g].astype(np.float64)
            for h in range(g * G, (g + 1) * G):
                q = Q[sl, h].astype(np.float64)
                s = np.where(seen, scale * (q @ k.T), -np.inf)
                e = np.exp(s - s.max(1, keepdims=True))
                e /= e.sum(1, keepdims=True)
                O[sl, h] = e @ v
                A[sl, h] = e @ np.abs(v)
                D[sl, h] = np.where(seen, np.abs(q) @ np.abs(k).T, 0).max(1)
    return O, A, D, N
