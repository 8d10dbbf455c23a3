"""Which keys the shared-prefix attention takes together, restated from its rules on the
host and in the kernel, so that a test can tell which path its inputs run."""
from __future__ import annotations

import numpy as np

OWN_ROWS, BLOCK, TILE, SETUP, JOIN = 48, 256, 64, 3, 4


def blocks(rows):
    return -(-rows // BLOCK)


def places(B, N, Hq, Hkv, D, groups, tokens):
    """Places of a launch by groups over prefixes of `tokens` tokens."""
    rows, prefix = N * Hq // Hkv, -(-tokens // TILE) + SETUP
    own = (-(-(tokens + N) // (4096 // D)) * 2 + 1 if rows <= OWN_ROWS
           else blocks(rows) * (prefix + -(-N // TILE)))
    return Hkv * ((blocks(B * rows) + groups) * prefix + B * own)


def by_groups(B, N, Hq, Hkv, D, groups, max_len, table_tokens):
    """The host's rule: whether the batch takes keys by groups at all."""
    rows = N * Hq // Hkv
    if groups == 0 or groups >= B or places(B, N, Hq, Hkv, D, groups, table_tokens) >= 1 << 30:
        return False
    if (B - groups) * Hkv * D * 4 * max_len < 32 << 20 or (blocks(rows) * BLOCK - rows) * 4 < blocks(rows) * BLOCK:
        return False
    together = blocks(B * rows)
    return rows <= OWN_ROWS or ((B * blocks(rows) - together) * (max_len // TILE)
                                > SETUP * together + JOIN * B * blocks(rows))


def shared_tiles(w, start, shared):
    """The kernel's rule: the tiles that each group takes together (ascending starts)."""
    G = w.Hq // w.Hkv
    nodes = np.full(w.B, w.N) if w.num_nodes is None else w.num_nodes
    out = []
    for s, n in enumerate(shared):
        b = [b for b in range(start[s], start[s + 1]) if nodes[b] > 0]
        if not b:
            out.append(0)
            continue
        tiles = max(min(n, int(w.kv_len[b].min())), 0) // TILE
        if w.N * G <= OWN_ROWS:
            out.append(tiles if len(b) > 1 else 0)
            continue
        apart, together = sum(blocks(int(nodes[i]) * G) for i in b), blocks(int(nodes[b].sum()) * G)
        out.append(tiles if (apart - together) * tiles > SETUP * together + JOIN * apart else 0)
    return out
