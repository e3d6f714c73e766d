"""Pages for a batch's requests (kv_reserve_paged) and rows by slot (kv_append_paged), as a
literal simulation: a Python list is the stack of free pages, requests are taken one by one.
The paper leaves the cache's management to the serving system (Limitations)."""
from __future__ import annotations

import numpy as np


def kv_reserve_paged(table, held, ctx_len, n_new, free_pages, n_free, page_rows, max_new):
    """Returns (table, held, free_pages, n_free, n_short, slots), all new."""
    B, max_pages = table.shape
    table, free_pages = table.copy(), free_pages.copy()
    num_pages = len(free_pages)
    stack = [int(x) for x in free_pages[:min(max(int(n_free), 0), num_pages)]]
    pushed_from = len(stack)
    have = [min(max(int(h), 0), max_pages) for h in held]
    ctx = [max(int(c), 0) for c in ctx_len]
    new = [min(max(int(n), 0), max_new) for n in n_new]
    want = [-(-(c + n) // page_rows) for c, n in zip(ctx, new)]
    short = [w > max_pages for w in want]
    for b in range(B):
        if not short[b]:
            stack += [int(p) for p in table[b, want[b]:have[b]]]
            have[b] = min(have[b], want[b])
    stack = stack[:num_pages]
    free_pages[pushed_from:len(stack)] = stack[pushed_from:]
    closed = False
    for b in range(B):
        if short[b] or want[b] <= have[b]:
            continue
        closed = closed or want[b] - have[b] > len(stack)
        if closed:
            short[b] = True
            continue
        while have[b] < want[b]:
            table[b, have[b]] = stack.pop()
            have[b] += 1
    slots = np.full((B, max_new), -1, dtype=np.int64)
    for b in range(B):
        if not short[b]:
            for i in range(new[b]):
                r = ctx[b] + i
                slots[b, i] = int(table[b, r // page_rows]) * page_rows + r % page_rows
    return table, np.array(have, np.int32), free_pages, len(stack), sum(short), slots


def kv_append_paged(K_new, V_new, slots, K_pages, V_pages):
    """The pools with row t of the new rows at slot slots[t]; other slots left out."""
    K, V = K_pages.copy(), V_pages.copy()
    pr, n = K.shape[1], K.shape[0] * K.shape[1]
    for t, s in enumerate(np.asarray(slots).reshape(-1)):
        if 0 <= s < n:
            K[s // pr, s % pr], V[s // pr, s % pr] = K_new[t], V_new[t]
    return K, V
