"""fp64 definitions of drafting over a part of a long cache: page bounds and scores, selection, sparse attention, token
weights, eviction.  Plain loops over numpy arrays, sharing nothing with the kernels.

Pools are [num_pages, hkv, P, D] arrays of numbers, page tables [C, max_pages], lengths [C].
"""
from __future__ import annotations

import math

import numpy as np


def pages_of(n, P):
    return -(-int(n) // P)


def rows_of(pool, table, c, n, h):
    """The first n rows [n, D] of KV head h of cache c (a contiguous cache: table None, pool [C, hkv, l_cap, D])."""
    if table is None:
        return pool[c, h, :n]
    P = pool.shape[2]
    return np.stack([pool[table[c, j // P], h, j % P] for j in range(n)]) if n else np.zeros((0, pool.shape[3]))


def page_bounds(k, table, lens, before, out):
    """out [num_pages, hkv, 2, D], changed where a page holds a token at or past before[c]."""
    out, P = out.copy(), k.shape[2]
    for c, n in enumerate(lens):
        for p in range(int(before[c]) // P, pages_of(n, P)):
            rows = k[table[c, p], :, :min(P, int(n) - p * P)]
            out[table[c, p], :, 0], out[table[c, p], :, 1] = rows.min(1), rows.max(1)  # (numpy's pass a NaN on)
    return out


def page_scores(q, bounds, table, lens, P, scale, out):
    """q [C, Nq, hq, D]; out [C, Nq, hkv, max_pages], changed for the caches' pages; and the sums of the products'
    magnitudes, which bound the rounding of a sum."""
    out, mag = out.copy(), np.zeros_like(out)
    hkv = out.shape[2]
    G = q.shape[2] // hkv
    for c, n in enumerate(lens):
        for p in range(pages_of(n, P)):
            lo, hi = bounds[table[c, p], :, 0], bounds[table[c, p], :, 1]
            for h in range(hkv):
                x = q[c, :, h * G:(h + 1) * G]
                terms = np.maximum(x * lo[h], x * hi[h])
                out[c, :, h, p] = scale * terms.sum(-1).max(-1)
                mag[c, :, h, p] = scale * (np.abs(x * lo[h]) + np.abs(x * hi[h])).sum(-1).max(-1)
    return out, mag


def select_top(scores, lens, rows_per_len, unit, keep, first, last):
    picks, counts = np.full((len(scores), keep), -1, np.int32), np.zeros(len(scores), np.int32)
    for r, s in enumerate(scores):
        n = pages_of(lens[r // rows_per_len], unit)
        m = min(n, keep)
        chosen = set(range(min(first, n))) | set(range(max(0, n - last), n))
        for i in sorted(range(n), key=lambda i: (0 if math.isnan(s[i]) else 1, -s[i] if not math.isnan(s[i]) else 0, i)):
            if len(chosen) >= m:
                break
            chosen.add(i)
        picks[r, :m], counts[r] = sorted(chosen), m
    return picks, counts


def line_of(parent, i):
    """Node i and its ancestors (parent None: a chain)."""
    out = [i]
    while True:
        i = i - 1 if parent is None else int(parent[i])
        if i < 0:
            return out
        out.append(i)


def attn_sparse(q, k, v, table, lens, picks, counts, draft_k, draft_v, parent, per_seq, N, scale):
    """out [C, Nq, hq, D], lse [C, Nq, hq]; the sums of p |v| [C, Nq, hq, D] and the largest sum of |q k| [C, Nq, hq]."""
    C, Nq, hq, D = q.shape
    hkv, P = k.shape[1], k.shape[2]
    G = hq // hkv
    out, lse = np.zeros(q.shape), np.zeros((C, Nq, hq))
    spread, mag = np.zeros(q.shape), np.zeros((C, Nq, hq))
    for c in range(C):
        for n in range(Nq):
            line = line_of(None if parent is None else parent[c // per_seq], N - Nq + n)
            for h in range(hkv):
                ks, vs = [draft_k[c, h, line]], [draft_v[c, h, line]]
                for p in picks[c, n, h, :counts[c, n, h]]:
                    rows = min(P, int(lens[c]) - p * P)
                    ks.append(k[table[c, p], h, :rows])
                    vs.append(v[table[c, p], h, :rows])
                ks, vs = np.concatenate(ks), np.concatenate(vs)
                for g in range(h * G, (h + 1) * G):
                    s = scale * (ks @ q[c, n, g])
                    top = s.max()
                    z = top + math.log(np.exp(s - top).sum())
                    w = np.exp(s - z)
                    out[c, n, g], lse[c, n, g], spread[c, n, g] = w @ vs, z, w @ np.abs(vs)
                    mag[c, n, g] = scale * (np.abs(ks) @ np.abs(q[c, n, g])).max()
    return out, lse, spread, mag


def key_weights(q, k, table, lens, lse, decay, weights, out, scale):
    """out [C, W], changed below the lengths; and the largest sum of |q k| that went into each."""
    out, mag = out.copy(), np.zeros_like(out)
    hq, hkv = q.shape[2], k.shape[1]
    for c, n in enumerate(lens):
        n = int(n)
        total = decay * weights[c, :n] if weights is not None and decay else np.zeros(n)
        for head in range(hq):
            rows = rows_of(k, table, c, n, head // (hq // hkv))
            for r in range(q.shape[1]):
                if lse[c, r, head] != -math.inf:
                    total = total + np.exp(scale * (rows @ q[c, r, head]) - lse[c, r, head])
                if n:
                    mag[c, :n] = np.maximum(mag[c, :n], scale * (np.abs(rows) @ np.abs(q[c, r, head])) + abs(lse[c, r, head])
                                            if lse[c, r, head] != -math.inf else 0)
        out[c, :n] = total
    return out, mag


def cache_evict(k, v, table, lens, kept, counts, weights, k_out, v_out, table_out, weights_out, free, free_count):
    """Arrays of any type; k_out and v_out may be k and v.  Returns everything that the call writes."""
    k, v, k_out, v_out = k.copy(), v.copy(), k_out.copy(), v_out.copy()
    weights_out, free, P = weights_out.copy(), free.copy(), k.shape[2]
    at = int(free_count)
    for c, m in enumerate(counts):
        for i in range(int(m)):
            j = int(kept[c, i])
            for src, dst in ((k, k_out), (v, v_out)):
                dst[table_out[c, i // P], :, i % P] = src[table[c, j // P], :, j % P]
            weights_out[c, i] = weights[c, j]
        weights_out[c, int(m):] = 0
        for p in range(pages_of(m, P), pages_of(lens[c], P)):
            free[at] = table[c, p]
            at += 1
    return k_out, v_out, np.asarray(counts).copy(), weights_out, free, at
