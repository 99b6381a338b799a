"""Plain CPU oracle of a serving step around the projections, in numpy float64 and Python integers.

TEST INFRASTRUCTURE ONLY. Only ``tests/``, the smoke check and the bench may import this module.
It shares no code with the GPU library (``paper_2607_19438_amd``) and imports nothing from it.

* ``kv_plan``: pages, slots and positions token by token;
* ``rope_frequencies`` / ``rope``: rotations as products with complex numbers of modulus ``gain``;
* ``quantise`` / ``encode_cache`` / ``decode_cache``: microscaled 4-bit blocks, every level compared;
* ``packed_attention`` / ``cached_attention``: ordinary softmax attention row by row over the keys that the row
  sees, with the magnitudes that the tolerance of ``attn_tolerance`` scales.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["kv_plan", "rope_frequencies", "rope", "rope_tolerance", "quantise", "encode_cache", "decode_cache",
           "gather_cache", "packed_attention", "cached_attention", "LEVELS"]

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def kv_plan(kv_len, q_len, table, free, page, T):
    """(cu_q, positions, slots, table, total_len, used); table is a changed copy."""
    table = np.array(table, dtype=np.int64, copy=True)
    cu, pos, slots, taken = [0], [0] * T, [-1] * T, 0
    for r, (n, m) in enumerate(zip(kv_len, q_len)):
        n, m = max(int(n), 0), max(int(m), 0)
        have, need = -(-n // page), -(-(n + m) // page)
        ids = {}
        for j in range(have, need):
            at = taken + j - have
            ids[j] = int(free[at]) if at < len(free) else -1
        for i in range(m):
            t, p = cu[-1] + i, n + i
            if t >= T:
                break
            j = p // page
            pos[t] = p
            if j < table.shape[1]:
                if j >= have and p % page == 0:
                    table[r, j] = ids[j]
                at = int(table[r, j]) if j < have else ids[j]
                if at >= 0 and at * page + p % page < 2 ** 31:
                    slots[t] = at * page + p % page
        taken += need - have
        cu.append(cu[-1] + m)
    total = [max(int(n), 0) + max(int(m), 0) for n, m in zip(kv_len, q_len)]
    return tuple(np.array(x, dtype=np.int64) for x in (cu, pos, slots, table, total, [taken]))


def rope_frequencies(rot, base, scaling="none", factor=1.0, low=1.0, high=4.0, length=1.0):
    out = []
    for i in range(rot // 2):
        f = math.exp(-2.0 * i / rot * math.log(base))
        if scaling == "none":
            w = 1.0
        elif scaling == "linear":
            w = 0.0
        elif scaling == "llama3":
            turns = length * f / (2 * math.pi)
            w = 0.0 if turns <= low else 1.0 if turns >= high else (turns - low) / (high - low)
        else:
            # the pair that makes t turns over the original context: length f = 2 pi t
            first = max(0, math.floor(rot / 2 * math.log(length / (2 * math.pi * high)) / math.log(base)))
            last = min(rot - 1, math.ceil(rot / 2 * math.log(length / (2 * math.pi * low)) / math.log(base)))
            width = last - first if last > first else 0.001
            w = 1.0 - min(1.0, max(0.0, (i - first) / width))
        out.append(w * f + (1 - w) * f / factor)
    return np.array(out), (0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0)


def rope(x, positions, inv_freq, rot_heads, interleaved=False, gain=1.0):
    """x [T][heads][D] -> float64, unrounded."""
    y = np.array(x, dtype=np.float64, copy=True)
    n = len(inv_freq)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None, :]
    turn = gain * np.exp(1j * np.mod(angle, 2 * np.pi))
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        z = (y[:, :rot_heads, a] + 1j * y[:, :rot_heads, b]) * turn[:, i, None]
        y[:, :rot_heads, a], y[:, :rot_heads, b] = z.real, z.imag
    return y


def rope_tolerance(x, y, inv_freq, rot_heads, interleaved=False, gain=1.0):
    """Half a bf16 step of the result (2^-8 of it), and for rotated elements 2^-20 of gain (|a| + |b|): the angle's
    turns are below a half and rounded to fp32 (2^-25 of a turn, 2^-22.3 in the sine), the sine and the cosine are
    good to about 2^-23, their product with the gain and the two products and the sum round at 2^-24 each."""
    x, tol = np.abs(np.asarray(x, dtype=np.float64)), 2.0 ** -8 * np.abs(y) + 1e-37
    n = len(inv_freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        s = (x[:, :rot_heads, a] + x[:, :rot_heads, b]) * abs(gain) * 2.0 ** -20
        tol[:, :rot_heads, a] += s
        tol[:, :rot_heads, b] += s
    return tol


def quantise(x):
    """Blocks [..., 32] -> (codes [..., 32], exponent bytes [...])."""
    x = np.asarray(x, dtype=np.float64)
    flat = x.reshape(-1, 32)
    codes = np.zeros(flat.shape, dtype=np.uint8)
    E = np.zeros(len(flat), dtype=np.uint8)
    for i, b in enumerate(flat):
        top = np.abs(b).max()
        if not np.isfinite(top):
            E[i] = 255
            continue
        e = -126
        if top > 0:
            p = math.floor(math.log2(top))
            while 2.0 ** p > top:
                p -= 1
            while 2.0 ** (p + 1) <= top:
                p += 1
            m = top / 2.0 ** p                       # 1 <= m < 2; to two significant bits: 1, 1.5 or 2
            e = min(max((p + 1 if m >= 1.75 else p) - 2, -126), 125)
        E[i] = e + 127
        a = np.abs(b) / 2.0 ** e
        d = np.abs(a[:, None] - LEVELS[None, :])
        near = d.min(axis=1)
        for j in range(32):
            best = [c for c in range(8) if d[j, c] == near[j]]
            codes[i, j] = next((c for c in best if c % 2 == 0), best[0]) | (8 if np.signbit(b[j]) else 0)
    return codes.reshape(x.shape), E.reshape(x.shape[:-1])


def dequantise(codes, E):
    s = np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]
    with np.errstate(over="ignore"):
        scale = np.where(E == 255, np.nan, 2.0 ** (E.astype(np.float64) - 127))
    return s * scale[..., None]


def encode_cache(k, v, page):
    """k, v [pages*page][Hkv][D] -> uint8 [pages][Hkv][page * (D + D/16)]."""
    n, Hkv, D = k.shape
    out = np.zeros((n // page, Hkv, page * (D + D // 16)), dtype=np.uint8)
    for which, x in enumerate((k, v)):
        codes, E = quantise(x.reshape(n, Hkv, D // 32, 32))
        codes = codes.reshape(n, Hkv, D)
        for s in range(n):
            p, o = divmod(s, page)
            c0 = (which * page + o) * (D // 2)
            out[p, :, c0:c0 + D // 2] = codes[s, :, 0::2] | (codes[s, :, 1::2] << 4)
            s0 = page * D + (which * page + o) * (D // 32)
            out[p, :, s0:s0 + D // 32] = E[s]
    return out


def decode_cache(cache, D):
    """(k, v) float64 [pages*page][Hkv][D]."""
    pages, Hkv, rec = cache.shape
    page = rec * 16 // (17 * D)
    out = []
    for which in range(2):
        x = np.zeros((pages, page, Hkv, D))
        for o in range(page):
            c0 = (which * page + o) * (D // 2)
            s0 = page * D + (which * page + o) * (D // 32)
            by = cache[:, :, c0:c0 + D // 2]
            codes = np.stack([by & 15, by >> 4], -1).reshape(pages, Hkv, D // 32, 32)
            x[:, o] = dequantise(codes, cache[:, :, s0:s0 + D // 32]).reshape(pages, Hkv, D)
        out.append(x.reshape(pages * page, Hkv, D))
    return out


def gather_cache(k, v, table_row, n, page):
    """The first n keys and values of a request; None where its table has no page for one."""
    idx = []
    for p in range(n):
        j = p // page
        at = int(table_row[j]) if j < len(table_row) else -1
        if at < 0 or (at + 1) * page > len(k):
            return None
        idx.append(at * page + p % page)
    return k[idx], v[idx]


def _row(q, k, v, scale):
    """q [D] over k, v [n][D], n >= 1."""
    s = (k @ q) * scale
    p = np.exp(s - s.max())
    return (p @ v) / p.sum(), (p @ np.abs(v)) / p.sum()


def packed_attention(q, k, v, cu, scale):
    """float64 arrays [T][H or Hkv][D] -> (o, absv); rows of no prompt are 0."""
    T, H, D = q.shape
    G = H // k.shape[1]
    o, a = np.zeros((T, H, D)), np.zeros((T, H, D))
    for c0, c1 in zip(cu[:-1], cu[1:]):
        for t in range(int(c0), int(c1)):
            for h in range(H):
                o[t, h], a[t, h] = _row(q[t, h], k[c0:t + 1, h // G], v[c0:t + 1, h // G], scale)
    return o, a


def cached_attention(q, k, v, table, kv_len, cu, page, scale):
    """k, v: decode_cache's. -> (o, absv); rows of no request are 0, those that need a missing page NaN."""
    T, H, D = q.shape
    G = H // k.shape[1]
    o, a = np.zeros((T, H, D)), np.zeros((T, H, D))
    for r in range(len(kv_len)):
        n = int(cu[r + 1] - cu[r])
        for i in range(n):
            seen = int(kv_len[r]) - n + i + 1
            if seen <= 0:
                continue
            got = gather_cache(k, v, table[r], seen, page)
            t = int(cu[r]) + i
            if got is None:
                o[t], a[t] = np.nan, np.nan
                continue
            for h in range(H):
                o[t, h], a[t, h] = _row(q[t, h], got[0][:, h // G], got[1][:, h // G], scale)
    return o, a
