"""Plain 64-bit definitions of what runs between the QKV projection and o_proj (test infrastructure only).

  kv_slots        pages, slots and positions of a step's tokens from the requests' lengths (whole numbers, loops)
  qk_norm_rope    RMSNorm of the heads and rotation by position, before any rounding to bf16
  attention       softmax attention over gathered keys, with the sums that tolerances are built from
"""
from __future__ import annotations

import math

import numpy as np


def kv_slots(cached, fresh, base, page, free, table, T):
    """Returns (row_off, kv_len, table, slots, positions, taken); table is a copy with the new pages filled in."""
    table = np.array(table, dtype=np.int64)
    R, cols = table.shape
    row_off, kv_len, slots, pos, taken = [0], [], [], [], 0
    for r in range(R):
        c, n = max(int(cached[r]), 0), max(int(fresh[r]), 0)
        have, want = -(-c // page), -(-(c + n) // page)
        for j in range(have, want):
            if j < cols:
                table[r, j] = free[taken] if taken < len(free) else -1
            taken += 1
        for at in range(c, c + n):
            p = table[r, at // page] if at // page < cols else -1
            slots.append(p * page + at % page if p >= 0 else -1)
            pos.append((0 if base is None else int(base[r])) + at)
        kv_len.append(c + n)
        row_off.append(row_off[-1] + n)
    slots, pos = slots[:T] + [-1] * (T - len(slots)), pos[:T] + [0] * (T - len(pos))
    return np.array(row_off), np.array(kv_len), table, np.array(slots), np.array(pos), taken


def qk_norm_rope(x, gamma, eps, inv_freq, axis, positions, interleaved, scale=1.0):
    """x: float64 [T, heads, D]; gamma float64 [D] or None; positions int [axes, T].  Returns (y, size): the turned heads
    and, per element, |y_a| + |y_b| of the pair it came from (what a rotation's rounding errors are relative to)."""
    T, _, D = x.shape
    y = x.astype(np.float64)
    if gamma is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * gamma
    n = len(inv_freq)
    ax = np.zeros(n, int) if axis is None else np.asarray(axis, int)
    out, size = y.copy(), np.abs(y)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        # the product of a 32-bit whole number and a 24-bit fraction is exact in long double, and so is its remainder
        ang = np.fmod(positions[ax[i]].astype(np.longdouble) * np.longdouble(inv_freq[i]), 2 * np.longdouble(math.pi) if np.finfo(np.longdouble).nmant < 60
                      else np.longdouble("6.283185307179586476925286766559005768"))
        c, s = np.cos(ang).astype(np.float64)[:, None] * scale, np.sin(ang).astype(np.float64)[:, None] * scale
        ya, yb = y[:, :, a], y[:, :, b]
        out[:, :, a], out[:, :, b] = ya * c - yb * s, yb * c + ya * s
        size[:, :, a] = size[:, :, b] = (np.abs(ya) + np.abs(yb)) * abs(scale)
    return out, size


def attention(q, keys, values, sees, scale):
    """One request's rows: q [n, Hk, G, D], keys / values [N, Hk, D], sees int [n]: how many keys of the list (its first
    ones) a row sees.  Returns (o, lse, absv, smax): softmax(scale q k) v, the log-sum-exp, sum p |v| per element, and
    the largest scale * sum |q_i k_i| among the keys a row sees."""
    n, Hk, G, D = q.shape
    N = keys.shape[0]
    o, lse = np.zeros((n, Hk, G, D)), np.full((n, Hk, G), -np.inf)
    absv, smax = np.zeros((n, Hk, G, D)), np.zeros((n, Hk, G))
    for h in range(Hk):
        k, v = keys[:, h], values[:, h]
        for i in range(n):
            m = min(int(sees[i]), N)
            if m <= 0:
                continue
            s = scale * (q[i, h] @ k[:m].T)
            top = s.max(-1, keepdims=True)
            e = np.exp(s - top)
            l = e.sum(-1, keepdims=True)
            p = e / l
            o[i, h], absv[i, h] = p @ v[:m], p @ np.abs(v[:m])
            lse[i, h] = (top + np.log(l))[:, 0]
            smax[i, h] = (scale * (np.abs(q[i, h]) @ np.abs(k[:m]).T)).max(-1)
    return o, lse, absv, smax
