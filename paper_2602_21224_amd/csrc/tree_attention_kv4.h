// What the two kernels of the attention over 4 bits share: how a workgroup finds its pieces
// of work, and the loads of codes.
#pragma once

#include "kv4.h"
#include "tree_attention_kernel.h"

namespace tv {
namespace {

// r / G for a row r < 2^11 of a sequence and KV head.
__device__ __forceinline__ int node_of(const Kv4AttnParams &p, int r) {
    return p.g_inv ? (int)__umulhi((unsigned)r, p.g_inv) : r;
}

// Tree tiles that row block rb of a sequence with `nodes` nodes visits: those up to its last
// row's node.
__device__ __forceinline__ int tree_tiles(const Kv4AttnParams &p, int rb, int nodes) {
    const int end = (rb + 1) * p.rows_per_block;
    return ((end >= nodes * p.G ? nodes : node_of(p, end - 1) + 1) + KT - 1) / KT;
}

// Virtual tiles of one KV head of a sequence: per row block the set-up tiles, ntp prefix
// tiles and its tree tiles.
__device__ __forceinline__ int head_tiles(const Kv4AttnParams &p, int ntp, int nodes) {
    int t = 0;
    for (int rb = 0; rb * p.rows_per_block < nodes * p.G; ++rb) t += p.setup_tiles + ntp + tree_tiles(p, rb, nodes);
    return t;
}
// Those of a sequence with a prefix of L tokens.
__device__ __forceinline__ int sequence_tiles(const Kv4AttnParams &p, int L, int nodes) {
    return p.Hkv * head_tiles(p, (L + KT - 1) / KT - span_of(L, p).gap, nodes);
}

// Contiguous shares of all units' virtual tiles, laid end to end as in tree_attention.hip:
// workgroup u takes [start_of(u), start_of(u + 1)), the first `more` of nw one tile more
// than the others' `each`. (Shares by 64-bit products and quotients took 10000 cycles to
// find a piece with.)
struct Shares {
    int nw, each, more;
    __device__ __forceinline__ Shares(int total, int num_wg) {
        nw = min(num_wg, total);
        each = nw > 0 ? total / nw : 0;
        more = total - each * nw;
    }
    __device__ __forceinline__ int start_of(int u) const { return min(u, nw) * each + min(u, more); }
    __device__ __forceinline__ int owner_of(int t) const {
        const int full = more * (each + 1);
        return t < full ? t / (each + 1) : more + (t - full) / each;
    }
};

// The part of a unit that a share covers: real tiles t0 .. t_end - 1 of its ulen, of which
// the first ntp are the prefix's.
struct Piece {
    int b, g, rb, L, nodes, rows_b, ntp, t0, t_end, ulen, slot;
    bool complete;
    Span sp;
    // Place of prefix tile t among all tiles of the prefix, or of tree tile t behind them.
    __device__ __forceinline__ int real(int t) const { return t >= sp.ns ? t + sp.gap : t; }
};

// The piece at virtual tile `pos` of the share [start, end) of workgroup w; moves pos past
// it. False if only set-up tiles of a unit are left there. The first call of a share writes
// the joining kernel's entry for the workgroup: the split unit whose last piece is its first.
__device__ __forceinline__ bool next_piece(const Kv4AttnParams &p, const Shares &sh, int w, int start, int end, int &pos,
                                           Piece &pc) {
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (g_cum[mid] <= pos) lo = mid; else hi = mid - 1;
    }
    pc.b = lo;
    pc.L = g_len[lo];
    pc.nodes = g_nn[lo];
    pc.rows_b = pc.nodes * p.G;
    pc.sp = span_of(pc.L, p);
    pc.ntp = (pc.L + KT - 1) / KT - pc.sp.gap;
    const int C = p.setup_tiles;
    const int per_g = (g_cum[lo + 1] - g_cum[lo]) / p.Hkv;
    int off = pos - g_cum[lo];
    pc.g = off / per_g;
    off -= pc.g * per_g;
    pc.rb = 0;
    pc.ulen = pc.ntp + tree_tiles(p, 0, pc.nodes);
    while (off >= C + pc.ulen) {
        off -= C + pc.ulen;
        ++pc.rb;
        pc.ulen = pc.ntp + tree_tiles(p, pc.rb, pc.nodes);
    }
    const int v_end = min(C + pc.ulen, off + (end - pos));
    const int unit_start = pos - off + C;              // share coordinate of the unit's real tile 0
    if (pos == start && threadIdx.x == 0) {
        const int wf = sh.owner_of(unit_start);
        const bool mine = unit_start < start && sh.owner_of(unit_start + pc.ulen - 1) == w;
        *reinterpret_cast<i32x4 *>(p.ws_desc + w * 4) =
            mine ? i32x4{pc.b, pc.g, pc.rb | (pc.nodes << 8), wf * 2 + (unit_start <= sh.start_of(wf) ? 0 : 1)}
                 : i32x4{-1, 0, 0, 0};
    }
    pos += v_end - off;
    pc.t0 = max(off - C, 0);
    pc.t_end = v_end - C;
    pc.complete = pc.t0 == 0 && pc.t_end == pc.ulen;
    pc.slot = w * 2 + (unit_start <= start ? 0 : 1);
    return pc.t_end > pc.t0;
}

// Whether the piece has a tile whose mask depends on the nodes' root paths.
__device__ __forceinline__ bool needs_paths(const Kv4AttnParams &p, const Piece &pc) {
    return pc.t_end > pc.ntp ||
           (pc.t_end > pc.sp.ns && pc.real(max(pc.t0, pc.sp.ns)) * KT < pc.sp.lo0 + p.N - 1);
}

// Row of the cache (of one KV head's tokens) that holds position pos on page id, or -1 if no
// node sees it: past the prefix, behind the window, or on a page that does not exist.
__device__ __forceinline__ long long row_of(const Kv4AttnParams &p, int head, int pos, int id, int L, const Span &sp) {
    const bool live = pos < L && (pos >= sp.lo || pos < sp.sinks) && (unsigned)id < (unsigned)p.num_pages;
    const long long row =
        (((long long)(unsigned)id * (unsigned)p.Hkv + (unsigned)head) << p.p_shift) + (unsigned)(pos & (p.P - 1));
    return live ? row : -1;
}

template <int N>
__device__ __forceinline__ void load_dwords(unsigned (&to)[N], const uint8_t *from) {
    static_assert(N == 2 || N == 4, "8 or 16 bytes");
    if constexpr (N == 4) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(from);
        to[0] = x[0]; to[1] = x[1]; to[2] = x[2]; to[3] = x[3];
    } else {
        const u32x2 x = *reinterpret_cast<const u32x2 *>(from);
        to[0] = x[0]; to[1] = x[1];
    }
}

// Keys that a row of node `node` sees of the prefix tile at position `base`.
__device__ __forceinline__ unsigned long long prefix_bits(const Kv4AttnParams &p, const Piece &pc, int base, int node) {
    const int lim = pc.L - base;
    unsigned long long x = lim >= KT ? ~0ull : (1ull << lim) - 1ull;
    if (!window_clear(pc.sp, base, p.N)) x &= window_bits(pc.sp, base, g_anc[node]);
    return x;
}

// Rows of padding nodes (not part of any unit): zeros with lse -inf, a few nodes per workgroup.
template <int D, int NT>
__device__ void clear_padding(const Kv4AttnParams &p, int w) {
    if (!p.num_nodes) return;
    const int chunks = p.Hq * D / 8;
    for (int idx = w; idx < p.B * p.N; idx += p.num_wg) {
        const int b = idx / p.N, i = idx - b * p.N;
        if (i < g_nn[b]) continue;
        u16x8 *op = reinterpret_cast<u16x8 *>(p.out + ((size_t)b * p.N + i) * p.Hq * D);
        for (int c = threadIdx.x; c < chunks; c += NT) op[c] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
        if (p.lse)
            for (int h = threadIdx.x; h < p.Hq; h += NT) p.lse[((size_t)b * p.N + i) * p.Hq + h] = kNegInf;
    }
}

}  // namespace
}  // namespace tv
