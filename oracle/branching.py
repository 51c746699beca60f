"""Plain 64-bit definitions of what a step does for requests with more than one continuation (test infrastructure only).

  tree_mask       ancestors and positions of drafted tokens from their parents (whole numbers, loops)
  attention       softmax attention in which every row has its own set of keys, with the sums that tolerances are built from
  token_logprobs  log probabilities, log-sum-exp, entropy and best alternatives of rows of logits
  kv_compact      accepted tokens moved together in one layer's cache
  kv_trim         pages given back
  kv_fork         rows of a page table forked
"""
from __future__ import annotations

import math

import numpy as np


def tree_mask(parents, row_off, base, words):
    """(bits bool [T][32 * words], positions [T])."""
    T = len(parents)
    bits, pos = np.zeros((T, 32 * words), bool), np.zeros(T, np.int64)
    for r in range(len(row_off) - 1):
        t0 = int(row_off[r])
        there = {}
        for i in range(int(row_off[r + 1]) - t0):
            p = int(parents[t0 + i])
            if i >= 32 * words or p < -1 or p >= i or (p >= 0 and p not in there):
                continue
            there[i] = (there[p] if p >= 0 else []) + [i]
            bits[t0 + i, there[i]] = True
            pos[t0 + i] = (0 if base is None else int(base[r])) + len(there[i]) - 1
    return bits, pos


def packed(bits):
    """bool [T][32 * words] as int32 [T][words], bit m % 32 of word m / 32."""
    T, n = bits.shape
    w = (bits.reshape(T, n // 32, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1)
    return w.astype(np.uint32).view(np.int32)


def attention(q, keys, values, sees, scale):
    """One request's rows: q [n, Hk, G, D], keys / values [N, Hk, D], sees bool [n, N].  Returns (o, lse, absv, smax) as the attention of
    oracle.serving does; keys that a row does not see may hold anything."""
    n, Hk, G, D = q.shape
    o, lse = np.zeros((n, Hk, G, D)), np.full((n, Hk, G), -np.inf)
    absv, smax = np.zeros((n, Hk, G, D)), np.zeros((n, Hk, G))
    for i in range(n):
        at = np.nonzero(sees[i])[0]
        if not len(at):
            continue
        for h in range(Hk):
            k, v = keys[at, h], values[at, h]
            s = scale * (q[i, h] @ k.T)
            top = s.max(-1, keepdims=True)
            with np.errstate(invalid="ignore"):
                e = np.exp(s - top)
                l = e.sum(-1, keepdims=True)
                o[i, h], absv[i, h] = e / l @ v, e / l @ np.abs(v)
                lse[i, h] = (top + np.log(l))[:, 0]
                smax[i, h] = (scale * (np.abs(q[i, h]) @ np.abs(k).T)).max(-1)
    return o, lse, absv, smax


def token_logprobs(x, ids, scale, k):
    """x float64 [T][V].  Returns (logprob [T][n_ids], lse [T], entropy [T], top_ids [T][k], top_logprobs [T][k])."""
    T, V = x.shape
    lp, lse, ent = np.zeros(np.shape(ids)), np.zeros(T), np.zeros(T)
    tid, tlp = np.full((T, k), -1, np.int64), np.full((T, k), -np.inf)
    for t in range(T):
        y = x[t] * scale
        with np.errstate(invalid="ignore", divide="ignore"):
            top = np.max(y) if not np.isnan(y).any() else math.nan
            if top == -math.inf:
                lse[t], ent[t], logp = -math.inf, 0.0, np.full(V, -math.inf)
            else:
                d = y - top
                ln = math.log(np.exp(d).sum()) if math.isfinite(top) else math.nan
                lse[t], logp = top + ln, d - ln      # (y - lse would lose ln where the logits are huge)
                p = np.exp(logp)
                ent[t] = -np.sum(np.where(p > 0, p * np.where(p > 0, logp, 0.0), 0.0)) if math.isfinite(top) else math.nan
        for j, i in enumerate(ids[t]):
            lp[t, j] = logp[i] if 0 <= i < V else -math.inf
        # by value, NaN last, then by index
        order = sorted(range(V), key=lambda i: (math.inf if np.isnan(x[t, i]) else -x[t, i] if x[t, i] != -math.inf else math.inf, np.isnan(x[t, i]), i)) if V <= 4096 else \
            np.lexsort((np.arange(V), -x[t]))
        for j, i in enumerate(order[:k]):
            tid[t, j], tlp[t, j] = i, logp[i]
    return lp, lse, ent, tid, tlp


def kv_compact(cache, row_off, kv_len, table, keep, n_keep):
    """cache [n_pages][page][...] of one layer.  Returns (cache afterwards, new_len)."""
    out, new_len = cache.copy(), []
    n_pages, page = cache.shape[:2]

    def place(r, at):
        if at < 0 or at // page >= table.shape[1] or not 0 <= table[r, at // page] < n_pages:
            return None
        return table[r, at // page], at % page
    for r in range(len(kv_len)):
        n = max(int(row_off[r + 1]) - int(row_off[r]), 0)
        ctx, last, kept = int(kv_len[r]) - n, -1, 0
        for d in range(min(int(n_keep[r]), keep.shape[1], n)):
            i = int(keep[r, d])
            if i <= last or i >= n:
                break
            a, b = place(r, ctx + i), place(r, ctx + d)
            if a is not None and b is not None:
                out[b] = cache[a]
            last, kept = i, kept + 1
        new_len.append(ctx + kept)
    return out, np.array(new_len)


def kv_trim(from_len, to_len, page, table, refs, n_pages):
    """Returns (table, refs, freed pages in rising order)."""
    table, refs, freed = table.copy(), None if refs is None else refs.copy(), set()
    for r in range(len(from_len)):
        for c in range(-(-max(int(to_len[r]), 0) // page), min(-(-max(int(from_len[r]), 0) // page), table.shape[1])):
            p, table[r, c] = int(table[r, c]), -1
            if not 0 <= p < n_pages:
                continue
            if refs is None:
                freed.add(p)
            elif refs[p] > 0:
                refs[p] -= 1
                if refs[p] == 0:
                    freed.add(p)
    return table, refs, np.array(sorted(freed), np.int64)


def kv_fork(src, dst, length, page, free, table, refs, n_pages):
    """Returns (table, refs, len, copies [n][3], taken)."""
    table, refs, length, taken, copies = table.copy(), None if refs is None else refs.copy(), length.copy(), 0, []
    R, cols = table.shape

    def hold(p):
        if refs is not None and 0 <= p < n_pages:
            refs[p] += 1
    old = table.copy()
    for a, b in zip(src, dst):
        copies.append([-1, -1, 0])
        if not (0 <= a < R and 0 <= b < R and a != b):
            continue
        n = min(max(int(length[a]), 0), cols * page)
        for c in range(n // page):
            table[b, c] = old[a, c]
            hold(old[a, c])
        if n % page:
            p = int(free[taken]) if taken < len(free) and 0 <= free[taken] < n_pages else -1
            taken += 1
            table[b, n // page] = p
            hold(p)
            t = int(old[a, n // page])
            if p >= 0 and 0 <= t < n_pages:
                copies[-1] = [t, p, n % page]
        length[b] = length[a]
    return table, refs, length, np.array(copies, np.int64).reshape(-1, 3), taken
