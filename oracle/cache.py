"""Oracle of the cache operators beside the attention (TEST INFRASTRUCTURE
ONLY): accumulated attention weights of cached keys, and eviction by them.

Plain numpy over one sequence, KV head and path row at a time: fp64 sums of
fp64 exponentials on exactly widened bf16 inputs, and an eviction that sorts
whole slots by (kind, weight, slot). Attention over shared prefixes is the
attention itself (`tree_attention`): sharing changes which keys are taken
together, not what is computed.
"""
from __future__ import annotations

import numpy as np

from .tree_build import bf16_bits_to_f32


def cached_rows(cache_bits, pages, n):
    """[n, Hkv, D] fp64: the first n positions' rows of one sequence."""
    P = cache_bits.shape[1]
    t = np.arange(n)
    return bf16_bits_to_f32(cache_bits[np.asarray(pages)[t // P], t % P]).astype(np.float64)


def accumulate_weights(q, lse, k_cache, page_table, kv_len, accept_idx, accept_len, weight,
                       position, seen, fixed_len=None, scale=0.0):
    """Returns (weight fp64, position) after adding, for every path row j that sees
    position t and every query head h of KV head g, exp(scale q.k_t - lse[j, h])."""
    B, N, Hq, D = q.shape
    Hkv = k_cache.shape[2]
    G = Hq // Hkv
    c = scale if scale > 0 else 1.0 / np.sqrt(D)
    weight = np.array(weight, dtype=np.float64)
    position = np.array(position)
    for b in range(B):
        L, n = int(kv_len[b]), int(accept_len[b])
        f = 0 if fixed_len is None else min(int(fixed_len[b]), L)
        if n == 0:
            continue
        k = cached_rows(k_cache, page_table[b], L + n)
        for h in range(Hq):
            g = h // G
            if h % G == 0:
                weight[b, g, L:L + n] = 0.0
                position[b, g, L:L + n] = int(seen[b]) + np.arange(n)
            for j in range(n):
                z = float(lse[b, accept_idx[b, j], h])
                if z == -np.inf:
                    continue
                row = bf16_bits_to_f32(q[b, accept_idx[b, j], h]).astype(np.float64)
                p = np.exp(c * (k[:L + j + 1, g] @ row) - z)
                weight[b, g, f:L + j + 1] += p[f:]
    return weight, position


def evict(weight, position, k_cache, v_cache, page_table, kv_len, seen, budget, recent=0,
          fixed_len=None):
    """Returns copies (weight, position, k_cache, v_cache, kept_len) after the eviction."""
    weight, position = np.array(weight), np.array(position)
    kc, vc = np.array(k_cache), np.array(v_cache)
    B, Hkv = weight.shape[:2]
    P = kc.shape[1]
    kept_len = np.zeros(B, dtype=np.int32)
    for b in range(B):
        L = int(kv_len[b])
        f = 0 if fixed_len is None else min(int(fixed_len[b]), L)
        keep = kept_len[b] = min(L, max(budget, f))
        for g in range(Hkv):
            def order(t):
                w = float(weight[b, g, t])
                kind = 0 if t < f else (1 if int(position[b, g, t]) >= int(seen[b]) - recent else 2)
                return (kind, 0 if np.isnan(w) else 1, 0.0 if np.isnan(w) else -w, t)
            kept = sorted(sorted(range(L), key=order)[:keep])
            holes = [t for t in range(keep) if t not in set(kept)]
            for dst, src in zip(holes, [t for t in kept if t >= keep]):
                weight[b, g, dst], position[b, g, dst] = weight[b, g, src], position[b, g, src]
                to = (page_table[b, dst // P], dst % P, g)
                at = (page_table[b, src // P], src % P, g)
                kc[to], vc[to] = k_cache[at], v_cache[at]
    return weight, position, kc, vc, kept_len
