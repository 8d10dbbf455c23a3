"""Inputs of the cache operators' tests: batches whose sequences share pages,
and weights, positions and accepted paths over a paged cache."""
from __future__ import annotations

import numpy as np

from paper_2602_21224_amd import workloads as W


def share_prefix(w, start, shared):
    """Point the page tables of every group's sequences at its first sequence's
    pages for the first shared[s] tokens (a multiple of the page size each).
    Every sequence of the group is at least that long."""
    for s, n in enumerate(shared):
        a, e = start[s], start[s + 1]
        assert n % w.P == 0 and (w.kv_len[a:e] >= n).all()
        w.page_table[a:e, :n // w.P] = w.page_table[a, :n // w.P]


def shared_workload(seed, *, B, N, Hq, Hkv, D, P, start, shared, own, ragged=False, depth=6,
                    tree="capped", poison=True):
    """A workload of groups start[s] .. start[s+1]-1 with shared[s] common tokens
    and own[0] .. own[1] more of its own per sequence."""
    rng = np.random.default_rng(seed)
    common = np.zeros(B, np.int64)
    for s, n in enumerate(shared):
        common[start[s]:start[s + 1]] = n
    lens = common + rng.integers(own[0], own[1] + 1, size=B)

    def fn(r):
        n = int(r.integers(0, N + 1)) if ragged else N
        if n == 0:
            return np.zeros(0, np.int32)
        return {"capped": lambda: W.tree_random_depth_capped(r, n, depth),
                "forest": lambda: W.tree_uniform_forest(r, n),
                "chain": lambda: W.tree_chain(n)}[tree]()
    w = W.make_workload("shared", seed, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, kv_len=lens, parent_fn=fn,
                        V=8, P=P, poison=poison, with_logits=False)
    share_prefix(w, start, shared)
    return w


def attention_bounds(oracle, w):
    """(out, lse, bound of |out error|) of the oracle. The products are exact and summed
    in fp32; each weight is rounded once to bf16 (half a step, 2^-8 of it), a partial
    result of a split row once more, and the output once: 2^-8 (2 sum p |v| + |out|),
    and 2^-12 of sum p |v| for the fp32 sums and exponentials."""
    a = (w.page_table, w.kv_len, w.parent)
    out, lse = oracle.tree_attention(w.q, w.k_tree, w.v_tree, w.k_cache, w.v_cache, *a,
                                     num_nodes=w.num_nodes)
    mag, _ = oracle.tree_attention(w.q, w.k_tree, w.v_tree & 0x7FFF, w.k_cache, w.v_cache & 0x7FFF,
                                   *a, num_nodes=w.num_nodes)
    return out, lse, 2.0 ** -8 * (2 * mag + np.abs(out)) + 2.0 ** -12 * mag


def lse_bound(D, scale_qk):
    """|lse error|: D products of fp32 sums, half a step (2^-24) each of sum |q_i k_i|
    <= |q||k|, and the fp32 exponentials and logarithm, some steps of the value."""
    return 2.0 ** -24 * ((D + 8) * scale_qk + 64)


def cache_state(seed, *, B, Hkv, D, P, lens, room=0, extra=40, fixed=0, poison=True, ties=False):
    """Paged K/V of random rows (slots no sequence holds are NaN), weights with a long
    tail, and positions as earlier evictions leave them: the fixed slots in order, then
    any distinct positions below `seen`."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    table, pages = W.paged_layout(rng, lens, room, P)
    k = W.f32_to_bf16_bits(rng.standard_normal((pages, P, Hkv, D), dtype=np.float32))
    v = W.f32_to_bf16_bits(rng.standard_normal((pages, P, Hkv, D), dtype=np.float32))
    if poison:
        W.poison_cache_tails(k, v, table, lens, P)
    T = table.shape[1] * P
    fx = np.minimum(np.full(B, fixed), lens).astype(np.int32)
    seen = (lens + rng.integers(0, extra + 1, size=B)).astype(np.int32)
    weight = (rng.random((B, Hkv, T)) ** 8 * 50).astype(np.float32)
    if ties:
        weight = np.floor(weight * 0.1).astype(np.float32)
    position = np.full((B, Hkv, T), -7, np.int32)
    for b in range(B):
        for g in range(Hkv):
            position[b, g, :fx[b]] = np.arange(fx[b])
            position[b, g, fx[b]:lens[b]] = fx[b] + rng.permutation(seen[b] - fx[b])[:lens[b] - fx[b]]
    return dict(k_cache=k, v_cache=v, page_table=table, kv_len=lens, seen=seen, fixed_len=fx,
                weight=weight, position=position)


def accepted_paths(rng, B, N, lens):
    """accept_idx [B, N] (ascending node ids, then -1) of the given lengths."""
    idx = np.full((B, N), -1, np.int32)
    for b in range(B):
        idx[b, :lens[b]] = np.sort(rng.choice(N, int(lens[b]), replace=False))
    return idx, np.asarray(lens, np.int32)
