"""Plain CPU oracle of the serving operators for many continuations and many tenants, in numpy float64 and Python integers.

TEST INFRASTRUCTURE ONLY. Only ``tests/``, the smoke check and the bench may import this module.
It shares no code with the GPU library (``paper_2607_19438_amd``) and imports nothing from it.

* ``shared_attention``: attention over the cache, each row by itself, with the shared keys of its group taken from the
  table of the group's first request that has rows;
* ``beam_values`` / ``beam_select``: every candidate's value, and the best of them by sorting;
* ``kv_reorder``: tables, copies and released pages entry by entry;
* ``adapters`` / ``adapter_tolerance``: row by row through the row's own adapter.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["shared_keys", "shared_attention", "beam_values", "beam_select", "beam_tolerance", "kv_reorder", "adapters", "adapter_tolerance"]


def shared_keys(kv_len, cu, groups, prefix, W, page):
    """[(first request that has rows, shared keys)] of the groups; (None, 0) where none has."""
    out = []
    for g in range(len(prefix)):
        has = [r for r in range(groups[g], groups[g + 1]) if cu[r + 1] > cu[r]]
        n = min([int(prefix[g]), W * page] + [max(int(kv_len[r]), 0) - int(cu[r + 1] - cu[r]) for r in has])
        out.append((has[0], max(n, 0) // 64 * 64) if has else (None, 0))
    return out


def shared_attention(q, k, v, table, kv_len, cu, groups, prefix, page, scale, rows=None):
    """k, v [pages*page][Hkv][D] -> (o, absv); rows of no request are 0, those that need a missing page NaN. ``rows``: of these
    only."""
    T, H, D = q.shape
    G = H // k.shape[1]
    table = np.asarray(table)
    lead = shared_keys(kv_len, cu, groups, prefix, table.shape[1], page)
    o, a = np.zeros((T, H, D)), np.zeros((T, H, D))
    for r in range(len(kv_len)):
        owner, common = next((lead[g] for g in range(len(prefix)) if groups[g] <= r < groups[g + 1]), (r, 0))
        n = int(cu[r + 1] - cu[r])
        for i in range(n):
            t, seen = int(cu[r]) + i, int(kv_len[r]) - n + i + 1
            if seen <= 0 or (rows is not None and t not in rows):
                continue
            slots = []
            for p in range(seen):
                row = table[owner if p < common else r]
                at = int(row[p // page]) if p // page < len(row) else -1
                slots.append(at * page + p % page if 0 <= at and (at + 1) * page <= len(k) else -1)
            if min(slots) < 0:
                o[t], a[t] = np.nan, np.nan
                continue
            for h in range(H):
                s = (k[slots, h // G] @ q[t, h]) * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                o[t, h], a[t, h] = w @ v[slots, h // G], w @ np.abs(v[slots, h // G])
    return o, a


def beam_values(logits, scores, finished, end):
    """Values [B][V] of one request's candidates, -inf for what is none."""
    B, V = logits.shape
    out = np.full((B, V), -np.inf)
    for b in range(B):
        if not scores[b] > -np.inf:
            continue
        if finished is not None and finished[b]:
            out[b, end] = scores[b]
            continue
        x = np.asarray(logits[b], dtype=np.float64)
        if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
            continue
        top = x.max()
        out[b] = float(scores[b]) + (x - (top + math.log(math.fsum(np.exp(x - top)))))
    return out


def beam_select(logits, scores, K, finished=None, end=0):
    """logits [R*B][V], scores [R][B] -> (scores float64, parents, tokens), each [R][K]. Equal values: the lower beam first, of a
    beam the larger logit, then the lower token."""
    R, B = scores.shape
    V = logits.shape[1]
    best, par, tok = np.full((R, K), -np.inf), np.full((R, K), -1), np.full((R, K), end)
    for r in range(R):
        val = beam_values(logits[r * B:(r + 1) * B], scores[r], None if finished is None else finished[r], end).ravel()
        order = np.arange(B * V), -np.asarray(logits[r * B:(r + 1) * B], dtype=np.float64).ravel(), np.arange(B * V) // V
        for k, i in enumerate(np.lexsort((*order, -val))[:K]):
            if val[i] > -np.inf:
                best[r, k], par[r, k], tok[r, k] = val[i], i // V, i % V
    return best, par, tok


def beam_tolerance(x, value):
    """How far a value of a row x of logits may be from its own. Each exp(x - top) of the sum is off by 2^-23 for the
    hardware's exponential and by 2 steps of 2^-24 of the exponent's size |x - top| (one for the product with log2 e, one
    for that constant); the differences are weighted with the terms, so the sum is off by
    (1 + mean |x - top|) 2^-23 of itself, and 16 of them are added in 32 bits at a time: 2^-20. The value is rounded once: 2^-24."""
    x = np.asarray(x, dtype=np.float64)
    d = x.max() - x[np.isfinite(x)]
    w = np.exp(-d)
    return 2.0 ** -20 + 2.0 ** -23 * (1.0 + (w * d).sum() / w.sum()) + 2.0 ** -24 * abs(value)


def kv_reorder(table, kv_len, parents, free, page, keep=None):
    """(new table, new lengths, src, dst, used, released) as lists and arrays of integers."""
    table = np.asarray(table, dtype=np.int64)
    R, B = np.asarray(parents).shape
    W = table.shape[1]
    new = np.full_like(table, -1)
    length, src, dst, used, released = [0] * (R * B), [-1] * (R * B), [-1] * (R * B), 0, []
    size = [max(int(n), 0) for n in kv_len]
    have = [min(-(-n // page), W) for n in size]
    for r in range(R):
        seen = set()
        for k in range(B):
            p = int(parents[r][k])
            if not 0 <= p < B:
                continue
            old, row = r * B + p, r * B + k
            length[row] = size[old]
            new[row, :have[old]] = table[old, :have[old]]
            if p in seen and size[old] % page:
                last = size[old] // page
                if used < len(free) and last < W:
                    src[row], dst[row] = int(table[old, last]), int(free[used])
                if last < W:
                    new[row, last] = free[used] if used < len(free) else -1
                used += 1
            seen.add(p)
        for j in range(0 if keep is None else max(int(keep[r]), 0), W):
            held = {int(new[r * B + k, j]) for k in range(B)}
            for b in range(B):
                at = int(table[r * B + b, j])
                if j < have[r * B + b] and at >= 0 and at not in held:
                    released.append(at)
                    held.add(at)
    return new, length, src, dst, used, released


def adapters(y, x, a, b, ids, gain=None, cu=None):
    """float64 arrays; returns the new y."""
    out = np.array(y, dtype=np.float64, copy=True)
    for r, i in enumerate(ids):
        if 0 <= i < len(a):
            for m in range(*((r, r + 1) if cu is None else (int(cu[r]), int(cu[r + 1])))):
                out[m] += (1.0 if gain is None else float(gain[i])) * (b[i] @ (a[i] @ x[m]))
    return out


def adapter_tolerance(y, x, a, b, ids, gain=None, cu=None):
    """Sums of n products in 32 bits are off by n 2^-23 of the sum of their sizes (a rounding or a cut at each addition): K and
    the gain's product in the inner sums, 3 r in the outer, and the addition to y once more."""
    K, r = x.shape[1], a.shape[1]
    tol = np.zeros(y.shape)
    for q, i in enumerate(ids):
        if 0 <= i < len(a):
            g = 1.0 if gain is None else abs(float(gain[i]))
            for m in range(*((q, q + 1) if cu is None else (int(cu[q]), int(cu[q + 1])))):
                s = g * (np.abs(b[i]) @ (np.abs(a[i]) @ np.abs(x[m])))
                tol[m] = (K + 3 * r + 4) * 2.0 ** -23 * s + 2.0 ** -23 * np.abs(y[m]) + 1e-37
    return tol
