"""CPU fp64 oracle of the 4-bit target cache: format, quantisation, page extension, windowed draft attention -- numpy.

TEST INFRASTRUCTURE ONLY.  Only tests, the package's ``smoke()`` self-check and
``bench.py``'s CPU-baseline leg may import it; the library never does, and
nothing here imports the library.

Not from the paper: a 4-bit KV cache is a compression variant of the target cache.  Definitions:
  e2m1   sign, 2 exponent bits e (bias 1), 1 mantissa bit m: e > 0 encodes (1 + m/2) 2^(e-1), e = 0 encodes m/2
  value  of a dim: e2m1(code) * e4m3(scale of its block of 16 dims) * 2^exp
  store  y = x 2^-exp, scale = e4m3(clip(max |y| / 6, 2^-9, 448)), code = e2m1(y / scale), nearest, ties to even,
         saturating; a NaN in a block makes its scale NaN
  group  16 tokens of one KV head, 2304 bytes: K codes [4 chunks of 32 dims][16 tokens][16 bytes], V codes, K scales
         [16 tokens][8 blocks], V scales; the even dim of a pair is a byte's low nibble
"""
from __future__ import annotations

import numpy as np

from .fp8 import e4m3_value

HEAD_DIM, BLOCK, TOKENS, BYTES = 128, 16, 16, 2304
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = e4m3_value(np.arange(0x7F))  # the non-negative finite numbers, ascending; index = code


def e2m1_value(codes) -> np.ndarray:
    """Decoded fp64 values of e2m1 codes 0..15, from the definition."""
    c = np.asarray(codes).astype(np.int64)
    e, m = (c >> 1) & 3, (c & 1).astype(np.float64)
    mag = np.where(e > 0, (1.0 + m / 2.0) * np.exp2(e - 1.0), m / 2.0)
    return np.where(c & 8, -mag, mag)


def nearest(x, grid) -> np.ndarray:
    """Index of the number of the ascending `grid` nearest to x >= 0, ties to the even index, saturating."""
    x = np.asarray(x, np.float64)
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = x - grid[lo], grid[hi] - x
    return np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)


def quantise(x, exp: int):
    """(codes [..., 128], scale bytes [..., 8]) of fp64 x [..., 128]."""
    x = np.asarray(x, np.float64)
    y = (x * 2.0 ** -exp).reshape(*x.shape[:-1], HEAD_DIM // BLOCK, BLOCK)
    bad = np.isnan(y).any(-1)
    top = np.where(bad, 0.0, np.abs(np.nan_to_num(y, nan=0.0, posinf=np.inf, neginf=-np.inf)).max(-1))
    # 6 times a grid point is exact, so the nearest scale to top / 6 is found without a division
    scale = np.maximum(nearest(np.minimum(top, 6 * 448.0), 6 * E4M3), 1)
    s = E4M3[scale][..., None]
    a = np.minimum(np.abs(np.where(np.isnan(y), 0.0, y)), 8 * s)
    code = _nearest_rows(a, s) + 8 * np.signbit(y)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 0x7F, scale).astype(np.uint8)


def _nearest_rows(a, s):
    """Index into E2M1 nearest to a / s, by comparing a with the products of s and the midpoints (all exact)."""
    code = np.zeros(a.shape, np.int64)
    for i in range(7):
        mid = s * (E2M1[i] + E2M1[i + 1]) / 2
        code += (a > mid) | ((a == mid) & (i % 2 == 1))
    return code


def values(codes, scales, exp: int) -> np.ndarray:
    """fp64 values of codes [..., 128] with scale bytes [..., 8]."""
    return e2m1_value(codes) * np.repeat(e4m3_value(scales), BLOCK, axis=-1) * 2.0 ** exp


def unpack(cache) -> tuple:
    """Codes and scales of K and V, token by token: cache uint8 [pages, hkv, page / 16, 2304] ->
    (k codes, k scales, v codes, v scales), [pages, hkv, page, 128] and [pages, hkv, page, 8]."""
    pages, hkv, groups, n = cache.shape
    assert n == BYTES
    out = []
    for kind in (0, 1):
        codes = np.zeros((pages, hkv, groups, TOKENS, HEAD_DIM), np.uint8)
        scales = np.zeros((pages, hkv, groups, TOKENS, HEAD_DIM // BLOCK), np.uint8)
        for t in range(TOKENS):
            for d in range(HEAD_DIM):
                byte = cache[..., 1024 * kind + (d // 32) * 256 + t * 16 + (d % 32) // 2]
                codes[..., t, d] = byte >> 4 if d % 2 else byte & 15
            scales[..., t, :] = cache[..., 2048 + 128 * kind + 8 * t:2048 + 128 * kind + 8 * t + 8]
        out += [codes.reshape(pages, hkv, groups * TOKENS, -1), scales.reshape(pages, hkv, groups * TOKENS, -1)]
    return tuple(out)


def pack(kc, ks, vc, vs) -> np.ndarray:
    """The inverse of unpack."""
    pages, hkv, page, _ = kc.shape
    cache = np.zeros((pages, hkv, page // TOKENS, BYTES), np.uint8)
    for kind, (c, s) in enumerate(((kc, ks), (vc, vs))):
        c = c.reshape(pages, hkv, page // TOKENS, TOKENS, HEAD_DIM)
        s = s.reshape(pages, hkv, page // TOKENS, TOKENS, HEAD_DIM // BLOCK)
        for t in range(TOKENS):
            for d in range(0, HEAD_DIM, 2):
                cache[..., 1024 * kind + (d // 32) * 256 + t * 16 + (d % 32) // 2] = c[..., t, d] | (c[..., t, d + 1] << 4)
            cache[..., 2048 + 128 * kind + 8 * t:2048 + 128 * kind + 8 * t + 8] = s[..., t, :]
    return cache


def extend(seq_lens, new_tokens, page_table, free_pages, free_count: int, page_size: int, max_tokens: int):
    """Page extension, one token after another.  Returns (lens, table, count, start, slots, caches, positions), or None
    where the call cannot be met."""
    table = np.array(page_table, np.int64)
    free = [int(x) for x in free_pages[:free_count]]
    lens, start = [], [0]
    slots, caches, pos = ([-1] * max_tokens for _ in range(3))
    t = 0
    for c, (length, new) in enumerate(zip(seq_lens, new_tokens)):
        if length < 0 or new < 0:
            return None
        for i in range(int(length), int(length) + int(new)):
            if i % page_size == 0:
                if i // page_size >= table.shape[1] or not free:
                    return None
                table[c, i // page_size] = free.pop()
            if t >= max_tokens:
                return None
            slots[t], caches[t], pos[t] = table[c, i // page_size] * page_size + i % page_size, c, i
            t += 1
        lens.append(int(length) + int(new))
        start.append(t)
    return (np.array(lens), table, len(free), np.array(start), np.array(slots), np.array(caches), np.array(pos))


def node_lines(parent, n: int) -> list:
    """For each draft node the nodes from it to its root; parent None: a chain."""
    lines = []
    for i in range(n):
        up = i - 1 if parent is None else int(parent[i])
        lines.append([i] + (lines[up] if up >= 0 else []))
    return lines


def visible(length: int, lines, node: int, window: int, sinks: int):
    """(target positions, draft nodes) that `node` sees."""
    at = lambda i: length + len(lines[i]) - 1  # noqa: E731
    sees = lambda p: window == 0 or at(node) - p < window or p < sinks  # noqa: E731
    return [j for j in range(length) if sees(j)], [a for a in lines[node] if sees(at(a))]


def attn(q, prefix_k, prefix_v, draft_k, draft_v, parent, window: int, sinks: int, scale: float):
    """One cache.  q [Nq, hq, 128]; prefix_k/v [hkv, L, 128]; draft_k/v [hkv, N, 128]; parent [N] or None.  All fp64.
    Returns out [Nq, hq, 128] and lse [Nq, hq]."""
    nq, hq, _ = q.shape
    hkv, length, _ = prefix_k.shape
    n = draft_k.shape[1]
    lines = node_lines(parent, n)
    out, lse = np.zeros(q.shape), np.zeros((nq, hq))
    for r in range(nq):
        js, ms = visible(length, lines, n - nq + r, window, sinks)
        for h in range(hq):
            kh = h // (hq // hkv)
            k = np.concatenate([prefix_k[kh][js], draft_k[kh][ms]])
            v = np.concatenate([prefix_v[kh][js], draft_v[kh][ms]])
            s = k @ q[r, h] * scale
            m = s.max()
            p = np.exp(s - m)
            out[r, h] = p @ v / p.sum()
            lse[r, h] = m + np.log(p.sum())
    return out, lse
