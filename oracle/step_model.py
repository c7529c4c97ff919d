"""The operators of include/emm_step.h in plain numpy and Python, in 64 bits: attention with a window and sinks, norms of heads with
rotation, and a step's page tables as a loop over the requests.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def window_attention(table, prefix, new, cu, q, k_pool, v_pool, page, window, sinks, scale, rows):
    """q [T][H][d], pools [pages][Hkv][page][d], float64.  Returns out, lse and the sum of p |v| (rows of no request: NaN).  Slots that no
    row of a request sees are not read; a slot that a row does not see has no part in the row, whatever it holds."""
    heads, kv_heads, d = q.shape[1], k_pool.shape[1], q.shape[2]
    g = heads // kv_heads
    out = np.full((rows, heads, d), np.nan)
    size = np.full((rows, heads, d), np.nan)
    lse = np.full((rows, heads), np.nan)
    for r, (c, m) in enumerate(zip(prefix, new)):
        c, m = int(c), int(m)
        if m == 0:
            continue
        low = max(0, c - window + 1)
        at = np.concatenate([np.arange(min(sinks, low)), np.arange(low, c + m)])
        pages, places = np.asarray(table[r])[at // page], at % page
        pos = c + np.arange(m)
        seen = (at[None] <= pos[:, None]) & ((pos[:, None] - at[None] < window) | (at[None] < sinks))
        rows_r = slice(int(cu[r]), int(cu[r]) + m)
        for h in range(kv_heads):
            k, v = k_pool[pages, h, places], v_pool[pages, h, places]
            odd = ~np.isfinite(v)
            clean = np.where(odd, 0.0, v)
            for e in range(h * g, (h + 1) * g):
                with np.errstate(invalid="ignore"):
                    s = np.where(seen, (q[rows_r, e] @ k.T) * scale, -np.inf)
                    top = s.max(axis=1, keepdims=True)
                    p = np.where(seen, np.exp(s - top), 0.0)
                    total = p.sum(axis=1, keepdims=True)
                    o = (p @ clean) / total
                    for key in np.flatnonzero(odd.any(axis=1)):
                        o[seen[:, key]] += np.where(odd[key], v[key], 0.0)
                    out[rows_r, e] = o
                    size[rows_r, e] = (p @ np.abs(clean)) / total
                    lse[rows_r, e] = top[:, 0] + np.log(total[:, 0])
    return out, lse, size


def norm_rope(x, weight, eps, angle, rotary, interleaved):
    """Rows x [T][heads][d]; angle [T][rotary / 2] or None; weight None: no norm.  float64."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if angle is not None:
        a = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, rotary // 2), slice(rotary // 2, rotary))
        cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
        p, q = x[..., a[0]].copy(), x[..., a[1]].copy()
        x[..., a[0]], x[..., a[1]] = p * cos - q * sin, q * cos + p * sin
    return x


def page_step(table, free_pages, count, lens, add, held, page, window, sinks, max_tokens):
    """The step's results as a dict of lists and arrays, named as in emm_page_step_params; the arguments stay as they are."""
    table, held, buffer = [list(map(int, row)) for row in table], list(map(int, held)), list(map(int, free_pages))
    free, width = buffer[:count], len(table[0]) if table else 0
    for r, c in enumerate(lens):
        held[r] = max(held[r], -(-sinks // page))
        while window and (held[r] + 1) * page <= c - window + 1:
            free.append(table[r][held[r]])
            held[r] += 1
    new, refused, enough = [], 0, True
    for r, (c, m) in enumerate(zip(lens, add)):
        c, m = int(c), max(int(m), 0)
        have, want = -(-c // page), -(-(c + m) // page)
        ok = c + m <= width * page
        if ok and want > have:
            enough = enough and want - have <= len(free)
            ok = enough
            for e in range(have, want if ok else have):
                table[r][e] = free.pop()
        new.append(m if ok else 0)
        refused += int(not ok and m > 0)
    buffer[count:max(count, len(free))] = free[count:]
    slots, positions = np.full(max_tokens, -1, np.int64), np.zeros(max_tokens, np.int32)
    at = 0
    for r, m in enumerate(new):
        for p in range(int(lens[r]), int(lens[r]) + m):
            slots[at], positions[at] = table[r][p // page] * page + p % page, p
            at += 1
    return {"page_table": table, "free_pages": buffer, "prefix_lens": list(map(int, lens)), "new_lens": new, "cu_new_lens": [0] + list(np.cumsum(new)),
            "lens_out": [int(c) + m for c, m in zip(lens, new)], "held_out": held, "free_count_out": [len(free)], "slots": slots,
            "positions": positions, "refused": [refused]}
