"""Packed prompts and the paged cache from their definitions, in numpy and 64 bits: one row, one token at a time."""
from __future__ import annotations

import numpy as np


def attend(q, k, v, scale):
    """One (sequence, query head): q [m, d] against k, v [n, d]; row i sees keys 0 .. n - m + i.
    Returns o [m, d], lse [m], weights [m, n]."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    m, n = len(q), len(k)
    o, lse, w = np.zeros((m, v.shape[1])), np.zeros(m), np.zeros((m, n))
    for i in range(m):
        see = n - m + i + 1
        s = scale * (k[:see] @ q[i])
        top = s.max()
        e = np.exp(s - top)
        w[i, :see] = e / e.sum()
        lse[i] = top + np.log(e.sum())
        o[i] = w[i, :see] @ v[:see]
    return o, lse, w


def attend_packed(q, keys_of, cu, n_kv_heads, scale):
    """q [T, Hq, d]; keys_of(b, h) -> k, v [n, d] of sequence b. Returns o [T, Hq, d], lse [T, Hq] and, per sequence, the
    weight that every key received [Hkv, n]."""
    T, Hq, _ = q.shape
    G = Hq // n_kv_heads
    o, lse, mass = np.zeros(q.shape), np.zeros((T, Hq)), []
    for b in range(len(cu) - 1):
        rows, per_head = slice(cu[b], cu[b + 1]), []
        for h in range(n_kv_heads if cu[b + 1] > cu[b] else 0):
            k, v = keys_of(b, h)
            got = np.zeros(len(k))
            for g in range(h * G, (h + 1) * G):
                o[rows, g], lse[rows, g], w = attend(q[rows, g], k, v, scale)
                got += w.sum(0)
            per_head.append(got)
        mass.append(np.array(per_head))
    return o, lse, mass


def slots(table_row, page_size, n):
    """Pool page and row of slots 0 .. n - 1."""
    j = np.arange(n)
    return table_row[j // page_size], j % page_size


def evict(mass, pos, n, seen, budget, sinks, recent):
    """One (sequence, KV head) with mass, pos [n]: the slots that go, ascending, and the moves (from, to)."""
    k = max(0, n - max(1, budget))
    bits = np.asarray(mass, dtype=np.float32).view(np.uint32)
    stays = [pos[j] < sinks or pos[j] >= seen - recent for j in range(n)]
    order = sorted(range(n), key=lambda j: (stays[j], 0 if stays[j] else int(bits[j]), int(pos[j]), j))
    out = sorted(order[:k])
    tail = [j for j in range(n - k, n) if j not in set(out)]
    return out, list(zip(tail, [j for j in out if j < n - k]))
