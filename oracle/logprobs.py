"""Log probabilities, ranks, entropy and top alternatives of a logits row (taps_logprobs), fp64."""
from __future__ import annotations

import math

import numpy as np


def logprobs_row(x, token, top):
    """x: a row's values (float64 holding the stored ones).  Returns (log probability, entropy,
    rank, top indices, their log probabilities, sum p |x - x_0| for error bounds)."""
    n = len(x)
    nan = np.isnan(x)
    # rank order: value descending, index ascending, NaN last
    order = np.lexsort((np.arange(n), np.where(nan, 0.0, -np.where(nan, 0.0, x)), nan))
    top_value = x[order[0]]
    w, d = np.zeros(n), np.zeros(n)
    if not math.isnan(top_value):
        same = x == top_value
        w[same] = 1.0
        with np.errstate(invalid="ignore"):
            below = ~same & ~nan & np.isfinite(x - top_value)
        d[below] = x[below] - top_value
        w[below] = np.exp(d[below])
    Z = w.sum()
    if Z == 0:
        lp = np.full(n, -np.inf)
        entropy = spread = 0.0
    else:
        lnz = math.log(Z)
        lp = np.where(w > 0, d - lnz, -np.inf)
        tiny = (w == 0) & (d < 0)                        # exp underflows, the logarithm does not
        lp[tiny] = d[tiny] - lnz
        spread = float((w * -d).sum() / Z)
        entropy = lnz + spread
    place = np.empty(n, dtype=np.int64)
    place[order] = np.arange(n)
    given = 0 <= token < n
    return (lp[token] if given else -np.inf, entropy, int(place[token]) if given else -1,
            order[:top].astype(np.int32), lp[order[:top]], spread)
