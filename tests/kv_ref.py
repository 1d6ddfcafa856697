"""The 4-bit cache's operators in plain numpy, 64 bits, one request at a time: what the tests hold the
HIP kernels to."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def quantise(x):
    """Codes and scale bytes of x [..., D] (finite), by trying every scale byte and every code."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(g).max(-1)
    byte = np.full(top.shape, 252)
    for s in range(252, 1, -1):
        byte = np.where(top <= 7 * 2.0 ** (s - 127), s, byte)
    y = g / 2.0 ** (byte[..., None] - 127.0)
    off = np.abs(np.abs(y)[..., None] - VALUES[:8])
    odd = np.arange(8) % 2
    code = np.argmin(off * 4 + 1e-9 * odd, -1)  # a tie between neighbours: the even code
    code = np.where(y < 0, code + 8, code)
    return code.reshape(x.shape), byte


def rounded(k, v):
    """Rows [rows][heads][D] of keys and values as the cache gives them back."""
    out = []
    bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
    for x, fill in ((k, np.nan), (v, 0.0)):
        code, byte = quantise(np.where(np.isfinite(x), x, 0.0))
        val = VALUES[code].reshape(byte.shape + (32,)) * 2.0 ** (byte[..., None] - 127.0)
        out.append(np.where(bad[..., None], fill, val.reshape(x.shape)))
    return out


class Cache:
    """Keys and values by (page, offset): [pages * page][heads][D] in 64 bits."""

    def __init__(self, pages, page, heads, D):
        self.page, self.k, self.v = page, np.zeros((pages * page, heads, D)), np.zeros((pages * page, heads, D))


def pack(cache, layers=1):
    """Bytes [layers][pages][heads * block] of a cache that holds values of the format (as rounded() gives)."""
    page, (slots, heads, D) = cache.page, cache.k.shape
    n = slots // page
    parts = []
    for x in (cache.k, cache.v):
        code, byte = quantise(np.where(np.isfinite(x), x, 0.0))
        byte = np.where(np.isnan(x).reshape(byte.shape + (32,)).any(-1), 255, byte)
        both = (code[..., 0::2] + 16 * code[..., 1::2]).astype(np.uint8)
        for a in (both, byte.astype(np.uint8)):
            parts.append(a.reshape(n, page, heads, -1).transpose(0, 2, 1, 3).reshape(n, heads, -1))
    one = np.concatenate(parts, -1).reshape(n, -1)
    return np.ascontiguousarray(np.broadcast_to(one, (layers,) + one.shape))


def plan(length, n, cap, page, max_blocks, free, held, table):
    """ts_kv_plan, literally: free is a list (the top last), held and table are changed in place."""
    R = len(length)
    rows = [min(int(x), cap - 1) for x in n]
    need = [-(-(max(int(length[q]), 0) + max(rows[q] + 1, 0)) // page) for q in range(R)]
    back = []
    for q in range(R):
        if need[q] <= max_blocks:
            for b in range(need[q], held[q]):
                back.append(int(table[q, b]))
                table[q, b] = -1
            held[q] = min(held[q], need[q])
    free += back[::-1]
    lack, granted, have = 0, np.full(R, -1, np.int32), list(free)
    for q in range(R):
        if need[q] > max_blocks:
            continue
        add = max(need[q] - int(held[q]), 0)
        lack += add
        if add and lack > len(have):
            continue
        for b in range(int(held[q]), need[q]):
            table[q, b] = free.pop()
        held[q] = need[q]
        granted[q] = max(rows[q], -1)
    slot = np.full((R, cap), -1, np.int32)
    for q in range(R):
        for i in range(granted[q] + 1):
            t = max(int(length[q]), 0) + i
            slot[q, i] = table[q, t // page] * page + t % page
    return slot, granted


def attention(q, k, v, sees, scale):
    """One request: q [rows][hq][D], k, v [tokens][heads][D], sees [rows][tokens].  Returns out, lse, the sum of
    w |v| / sum w (what rounding a weight can move) and, per row and head, the largest sum of |q||k| * scale."""
    rows, hq, D = q.shape
    group = hq // k.shape[1]
    out, lse = np.zeros((rows, hq, D)), np.full((rows, hq), -np.inf)
    mass, mag = np.zeros((rows, hq, D)), np.zeros((rows, hq))
    for i in range(rows):
        t = np.flatnonzero(sees[i])
        if not len(t):
            continue
        for a in range(hq):
            kk, vv = k[t, a // group], v[t, a // group]
            s = kk @ q[i, a] * scale
            mag[i, a] = np.abs(scale) * np.nanmax(np.abs(kk) @ np.abs(q[i, a])) if not np.isnan(s).all() else np.nan
            w = np.exp(s - s.max())
            out[i, a] = w @ vv / w.sum()
            mass[i, a] = w @ np.abs(vv) / w.sum()
            lse[i, a] = s.max() + np.log(w.sum())
    return out, lse, mass, mag


def sees(length, rows, total, mask_rows=None):
    """[rows][total]: the context, and of the new rows those of the mask's bits (or a chain's)."""
    s = np.zeros((rows, total), bool)
    s[:, :length] = True
    for i in range(rows):
        for j in range(rows):
            if length + j < total:
                s[i, length + j] = j <= i if mask_rows is None else mask_rows[i, j // 32] >> (j % 32) & 1
    return s


def tree_bits(parent, rows, words):
    """Mask words of a tree's rows, as ts_tree_mask gives them."""
    bits = np.zeros((rows, words), np.uint32)
    for i in range(rows):
        a = i
        while a >= 0:
            bits[i, a // 32] |= np.uint32(1 << (a % 32))
            a = parent[a]
    return bits
