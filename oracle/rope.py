"""Per-head RMSNorm, rotary positions and the cache write of new rows (qk_rope_paged), fp64."""
from __future__ import annotations

import numpy as np

from .pages import kv_append_paged


def rope_frequencies(rot_dim, theta, scaling="none", factor=1.0, trained_len=1):
    """Turns per position (radians) of each pair, and the factor of cosines and sines."""
    freqs = []
    for pair in range(rot_dim // 2):
        base = theta
        if scaling == "ntk":
            base = theta * factor ** (rot_dim / (rot_dim - 2))
        f = 1.0 / base ** (2 * pair / rot_dim)
        if scaling == "linear":
            f = f / factor
        if scaling == "yarn":
            turns = trained_len / (2 * np.pi / f)
            keep = 0.0 if turns < 1 else 1.0 if turns > 32 else (turns - 1) / 31
            f = keep * f + (1 - keep) * f / factor
        freqs.append(f)
    return np.array(freqs), 1 + 0.1 * np.log(factor) if scaling == "yarn" else 1.0


def rms_norm(x, w, eps):
    """x [..., hd]; w None: x itself."""
    if w is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def rotate(x, positions, freqs, mscale, interleaved):
    """x [rows][heads][hd], pair by pair."""
    y = x.copy()
    half = len(freqs)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        ang = positions.astype(np.float64) * freqs[j]
        c, s = (mscale * np.cos(ang))[:, None], (mscale * np.sin(ang))[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def qk_rope_paged(Q, K, V, positions, slots, freqs, mscale, interleaved, q_norm, k_norm, eps,
                  K_pages, V_pages):
    """Returns the queries and the pools, all fp64, and for error bounds the normed values'
    magnitude sums |a| + |b| of each value's pair (|x| outside the rotation)."""
    def ready(x, w):
        n = rms_norm(x.astype(np.float64), w, eps)
        mag = np.abs(rotate(np.abs(n), np.zeros(len(x)), freqs, 1.0, interleaved))
        half = len(freqs)
        for j in range(half):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            mag[..., a] = mag[..., b] = np.abs(n[..., a]) + np.abs(n[..., b])
        return rotate(n, positions, freqs, mscale, interleaved), mag
    Qr, Qm = ready(Q, q_norm)
    Kr, Km = ready(K, k_norm)
    Kp, Vp = kv_append_paged(Kr, V.astype(np.float64), slots, K_pages.astype(np.float64),
                             V_pages.astype(np.float64))
    Kmag, _ = kv_append_paged(Km, Km, slots, np.zeros_like(Kp), np.zeros_like(Kp))
    return Qr, Kp, Vp, Qm, Kmag
