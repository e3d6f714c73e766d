"""Attention of one new token per request over a paged cache (decode_attn_paged), fp64."""
from __future__ import annotations

import numpy as np


def decode_attention_paged(Q, K_pages, V_pages, table, kv_len, scale):
    """Q [B][Hq][hd]; returns O [B][Hq][hd] and, for error bounds, the sums of the weighted
    |v| per output and the largest sum_d |q_d k_d| per query head."""
    B, Hq, hd = Q.shape
    pr, Hkv = K_pages.shape[1], K_pages.shape[2]
    G = Hq // Hkv
    O, A, D = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros((B, Hq))
    for b in range(B):
        n = int(kv_len[b])
        if n == 0:
            continue
        r = np.arange(n)
        pages, at = table[b, r // pr], r % pr
        k, v = K_pages[pages, at].astype(np.float64), V_pages[pages, at].astype(np.float64)
        for h in range(Hq):
            q = Q[b, h].astype(np.float64)
            s = scale * (k[:, h // G] @ q)
            e = np.exp(s - s.max())
            e /= e.sum()
            O[b, h] = e @ v[:, h // G]
            A[b, h] = e @ np.abs(v[:, h // G])
            D[b, h] = np.max(np.abs(k[:, h // G]) @ np.abs(q))
    return O, A, D
