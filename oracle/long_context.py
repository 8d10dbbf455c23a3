"""Oracle of the operators for long contexts (TEST INFRASTRUCTURE ONLY): a cache held in
4 bits, and tree attention inside a sliding window.

Plain numpy: the code of a value is the nearest of the representable ones, found by
distance, and the attention walks each node's root path and each head's keys in fp64.
"""
from __future__ import annotations

import numpy as np

from .tree_build import bf16_bits_to_f32

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize4(bits):
    """(codes [..., D/2] uint8, scale bytes [..., D/32] uint8) of bf16 rows [..., D]."""
    with np.errstate(invalid="ignore"):         # signalling NaNs
        x = bf16_bits_to_f32(bits).astype(np.float64)
    blocks = x.reshape(-1, 32)
    top = np.abs(blocks).max(1)
    bad = ~np.isfinite(blocks).all(1)
    top[bad] = 0.0
    e = np.full(len(blocks), -126)
    while (more := (top > 7 * 2.0 ** e) & (e < 125)).any():
        e += more
    y = np.where(bad[:, None], 0.0, blocks) / 2.0 ** e[:, None]
    codes = np.zeros(blocks.shape, np.uint8)
    best = np.full(blocks.shape, np.inf)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):           # a tie lies between an even and an odd code: even first
        d = np.abs(np.abs(y) - GRID[c])
        codes[d < best] = c
        best = np.minimum(best, d)
    codes = (codes + 8 * (np.signbit(y) & ~bad[:, None])).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    codes = codes.reshape(x.shape)
    return codes[..., 0::2] + 16 * codes[..., 1::2], scales.reshape(x.shape[:-1] + (x.shape[-1] // 32,))


def dequantize4(codes, scales):
    """fp64 rows [..., D] of codes [..., D/2] and scale bytes [..., D/32]."""
    n = np.stack([codes & 15, codes >> 4], axis=-1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    v = GRID[n & 7] * np.where(n & 8, -1.0, 1.0)
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(power, 32, axis=-1)


def write4(k, v, k4, v4, scales, page_table, start, idx=None, count=None):
    """Copies (k4, v4, scales) of the cache after the write, and the held rows (k, v) fp64
    (zeros where nothing was written)."""
    k4, v4, scales = np.array(k4), np.array(v4), np.array(scales)
    B, T, Hkv, D = k.shape
    P = k4.shape[2]
    held = [np.zeros(k.shape), np.zeros(k.shape)]
    for b in range(B):
        n = T if count is None else min(max(int(count[b]), 0), T)
        for j in range(n):
            src = j if idx is None else int(idx[b, j])
            pos = int(start[b]) + j
            page = page_table[b, pos // P]
            for i, (rows, codes) in enumerate(((k, k4), (v, v4))):
                c, e = quantize4(rows[b, src])
                codes[page, :, pos % P] = c
                scales[page, :, pos % P, i] = e
                held[i][b, j] = dequantize4(c, e)
    return k4, v4, scales, held[0], held[1]


def visible(parent, L, n, window, sinks):
    """For each of n nodes: (prefix positions, path nodes) that it sees."""
    depth, rows, t = [], [], np.arange(L)
    for i in range(n):
        p = int(parent[i])
        depth.append(0 if p < 0 else depth[p] + 1)
        at = L + depth[i]
        path, a = [], i
        while a >= 0:
            path.append(a)
            a = int(parent[a])
        if window == 0:
            rows.append((t, path[::-1]))
        else:
            rows.append((t[(t < sinks) | (t > at - window)],
                         [a for a in path[::-1] if L + depth[a] < sinks or L + depth[a] > at - window]))
    return rows


def window_attention(q, k_tree, v_tree, k_rows, v_rows, page_table, kv_len, parent, window, sinks, num_nodes=None,
                     scale=0.0):
    """(out, lse, sum of weight times |v|), fp64. k_rows(pages, slots) gives cached rows
    [n, Hkv, D] fp64, so that the cache may be held in any form."""
    B, N, Hq, D = q.shape
    Hkv = k_tree.shape[2]
    G = Hq // Hkv
    P = k_rows.P
    c = scale if scale > 0 else 1.0 / np.sqrt(D)
    out, mag = np.zeros((B, N, Hq, D)), np.zeros((B, N, Hq, D))
    lse = np.full((B, N, Hq), -np.inf)
    for b in range(B):
        n = N if num_nodes is None else int(num_nodes[b])
        for i, (pos, path) in enumerate(visible(parent[b], int(kv_len[b]), n, window, sinks)):
            pages, slots = page_table[b, pos // P], pos % P
            k = np.concatenate([k_rows(pages, slots), bf16_bits_to_f32(k_tree[b, path]).astype(np.float64)])
            v = np.concatenate([v_rows(pages, slots), bf16_bits_to_f32(v_tree[b, path]).astype(np.float64)])
            qi = bf16_bits_to_f32(q[b, i]).astype(np.float64)
            for h in range(Hq):
                s = c * (k[:, h // G] @ qi[h])
                m = s.max()
                w = np.exp(s - m)
                lse[b, i, h] = m + np.log(w.sum())
                w /= w.sum()
                out[b, i, h] = w @ v[:, h // G]
                mag[b, i, h] = w @ np.abs(v[:, h // G])
    return out, lse, mag


class Rows16:
    """Cached rows of a bf16 cache [num_pages, P, Hkv, D]."""

    def __init__(self, bits):
        self.bits, self.P = bits, bits.shape[1]

    def __call__(self, pages, slots):
        return bf16_bits_to_f32(self.bits[pages, slots]).astype(np.float64)


class Rows4:
    """Cached rows of a cache in 4 bits; `which`: 0 for K, 1 for V."""

    def __init__(self, codes, scales, which):
        self.codes, self.scales, self.which, self.P = codes, scales, which, codes.shape[2]

    def __call__(self, pages, slots):
        return dequantize4(self.codes[pages, :, slots], self.scales[pages, :, slots, self.which])
