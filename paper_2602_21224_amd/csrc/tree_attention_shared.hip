// Tree-masked attention for batches whose sequences share a prefix, for gfx950
// (MI355X): the attention of tree_attention.hip, whose tiles, ring, periods and
// pieces it uses, with the shared keys taken for all rows of a group at once.
//
//   * The keys of a group's shared prefix are units of their own, over the
//     query rows of all its sequences at once: rows of a group are its
//     sequences' real nodes one after another, in blocks of 256 as above, so a
//     shared K/V tile is read once per row block of the group instead of once
//     per row block of every sequence. What each sequence has behind the shared
//     tiles (its own prefix and its tree) are units as before. Both kinds are
//     laid end to end and shared out together.
//   * How many keys are taken together is the kernel's choice: whole tiles, at
//     most what the shortest sequence of the group has, so shared tiles need no
//     mask and the sequences' own tiles start at a tile. Results do not depend
//     on it beyond rounding. A group whose rows fill hardly fewer blocks together
//     than its sequences' blocks, each by itself, takes none: every block visits
//     every tile once either way, and rows of one piece need no joining.
//   * Every row of such a group has two results to be joined, one per kind. A
//     unit that one workgroup covers leaves whole normalised rows and their
//     log-sum-exps, a split unit leaves pieces as above and a record of the
//     workgroups that hold them; a second kernel joins them row by row. Every row
//     of such a batch is joined, and rounding both its parts to bf16 took the
//     error of the result from 0.0023 to 0.0028 of it (0.0017 is the rounding of
//     the output itself): parts are fp16 with a power of two per row instead,
//     half a step 2^-11 of them, for the same bytes (in fp32 a batch of 16
//     sequences x 12 rows x 32 heads took 53 us instead of 47).
//
// Kernel times, attention and joining: decoding 64 sequences x 32 heads over 4096 shared
// tokens and up to 512 of their own 27 + 7 us (plain call 145-180; 87 MB without
// repetition, 18 us of a large copy), 16 sequences x 12 nodes x 32 KV heads over 1024 shared
// and up to 1024 own tokens 37-46 + 8 us (plain 85; 157 MB, 33 us). Fill and drain, the joining
// launch and the shares' own unevenness are what is left.
#include "tree_attention_common.h"

namespace tv {
namespace {

constexpr int NW = 8;                    // waves of a workgroup
constexpr int NT = NW * kWave;

// Work tables. "Virtual sequence" v < groups is the shared prefix of group v,
// groups + b what sequence b has of its own.
__shared__ int g_vcum[kMaxGroups + kMaxBatchShared + 1];
__shared__ int g_slen[kMaxBatchShared];          // clamped prefix length per sequence
__shared__ int g_ncum[kMaxBatchShared + 1];      // real nodes of the sequences before b
__shared__ int g_gtiles[kMaxGroups];             // tiles taken together (first: shortest prefix of the group)
__shared__ int g_first[kMaxGroups];              // first sequence that has nodes
__shared__ int g_blocks[kMaxGroups];             // row blocks of the sequences, each by itself
__shared__ unsigned short g_gstart[kMaxGroups + 1];
__shared__ unsigned short g_group[kMaxBatchShared];       // group of a sequence, or kMaxGroups

// Query rows per KV head of group s: those of its sequences' real nodes.
__device__ __forceinline__ int group_rows(int s, const SharedAttnParams &p) {
    return (g_ncum[g_gstart[s + 1]] - g_ncum[g_gstart[s]]) * p.G;
}

// Prefix tiles of sequence b that its group takes together.
__device__ __forceinline__ int shared_tiles_of(int b) {
    const int s = g_group[b];
    return s < kMaxGroups ? g_gtiles[s] : 0;
}

template <int D>
struct OwnGeo {
    static constexpr int kKeys = own_keys(D);          // per tile
    static constexpr int kLoads = 8;                   // 1 KB loads of K (and of V) per tile
    static constexpr int kKeysPerLoad = 512 / D;
    static constexpr int kHalfBytes = 8192;            // of K, and of V
};

// Time of a (virtual) tile of the shared units, which is bound by its products, in
// places of own units, whose tiles are bound by their loads and, of several row tiles,
// by their latency: what divides the workgroups between the two. us per call with 2, 3
// and 4 own tiles per shared one: head size 128, 16 rows: 64 sequences of one row over
// 4096 shared tokens 40.0, 35.3, 33.4, 16 of 8 rows over 16384 57.5, 55.6, 58.4, of 12
// rows over 1024 56.9, 49.4, 49.7; 32 rows 39.0, 38.5, 41.3; 48 rows 44.2, 47.8, 49.1;
// head size 64: 27.1, 24.9, 26.2 and 26.1, 24.7, 25.4.
template <int D, int RT>
constexpr int shared_tile_cost() {
    return D == 64 ? 3 * kOwnTile : RT == 1 ? 7 * kOwnTile / 2 : 2 * kOwnTile;
}

// Real tiles of a sequence's units: prefix positions from `from` on, then the nodes.
template <int D>
__device__ __forceinline__ int own_tiles(int L, int from, int nodes) {
    return nodes == 0 ? 0 : (L - from + nodes + OwnGeo<D>::kKeys - 1) / OwnGeo<D>::kKeys;
}

// The tables of a batch with shared prefixes, by all threads; w = 0 leaves what
// the joining kernel needs of them in the workspace. D_OWN > 0: the sequences' own
// keys are units of tree_attention_own.h for that head size.
template <int D_OWN>
__device__ void build_shared_tables(const SharedAttnParams &p, int w) {
    static_assert(NT >= kMaxGroups, "one thread per group");
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const int promised = tid < p.groups ? p.shared_len[tid] : 0;    // asked for early
    if (tid < kWave) {
        int top = 0;                     // a start counts as the largest before it
        for (int s0 = 0; s0 <= p.groups && p.groups > 0; s0 += kWave) {
            const int s = s0 + lane;
            const int x = s <= p.groups ? min(max(p.group_start[s], 0), p.B) : 0;
            const int y = max(top, wave_prefix_max(x));
            if (s <= p.groups) g_gstart[s] = (unsigned short)y;
            top = __shfl(y, kWave - 1);
        }
    } else if (tid < 2 * kWave) {
        int carry = 0;
        for (int b0 = 0; b0 < p.B; b0 += kWave) {
            const int b = b0 + lane;
            const int n = b < p.B ? nodes_of(b, p) : 0;
            const int x = wave_prefix_sum(n);
            if (b < p.B) {
                g_ncum[b] = carry + x - n;
                g_slen[b] = clamp_len(p.kv_len[b], p);
            }
            carry += __shfl(x, kWave - 1);
        }
        if (lane == 0) g_ncum[p.B] = carry;
    }
    if (tid < p.groups) {
        g_gtiles[tid] = 0x7FFFFFFF;
        g_first[tid] = 0x7FFFFFFF;
        g_blocks[tid] = 0;
    }
    __syncthreads();
    for (int b = tid; b < p.B; b += NT) {
        int s = kMaxGroups;
        if (p.groups > 0 && b >= g_gstart[0] && b < g_gstart[p.groups]) {
            int lo = 0, hi = p.groups - 1;           // the last group that starts at or before b
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (g_gstart[mid] <= b) lo = mid; else hi = mid - 1;
            }
            s = lo;
        }
        g_group[b] = (unsigned short)s;
        if (s < kMaxGroups && g_ncum[b + 1] > g_ncum[b]) {
            atomicMin(&g_gtiles[s], g_slen[b]);
            atomicMin(&g_first[s], b);
            atomicAdd(&g_blocks[s], D_OWN ? 1 : row_blocks_of((g_ncum[b + 1] - g_ncum[b]) * p.G, p));
        }
    }
    __syncthreads();
    if (tid < p.groups) {
        const int tiles = max(min(g_gtiles[tid], promised), 0) / KT;
        const int apart = g_blocks[tid], together = row_blocks_of(group_rows(tid, p), p);
        const bool pays = D_OWN ? apart > 1
                                : (apart - together) * tiles > p.setup_tiles * together + kJoinTiles * apart;
        g_gtiles[tid] = pays ? tiles : 0;
    }
    __syncthreads();
    if (tid < kWave) {
        int carry = 0;
        const int nv = p.groups + p.B;
        for (int v0 = 0; v0 < nv; v0 += kWave) {
            const int v = v0 + lane;
            int t = 0;
            if (v < p.groups) {
                if (g_gtiles[v] > 0)
                    t = p.Hkv * row_blocks_of(group_rows(v, p), p) * (p.setup_tiles + g_gtiles[v]);
            } else if (v < nv) {
                const int b = v - p.groups, n = g_ncum[b + 1] - g_ncum[b];
                if constexpr (D_OWN > 0) {
                    const int own = own_tiles<D_OWN>(g_slen[b], shared_tiles_of(b) * KT, n);
                    t = own > 0 ? p.Hkv * (own * kOwnTile + 1) : 0;
                } else {
                    t = p.Hkv * tiles_per_head((g_slen[b] + KT - 1) / KT - shared_tiles_of(b), n * p.G, p);
                }
            }
            const int x = wave_prefix_sum(t);
            if (v < nv) g_vcum[v] = carry + x - t;
            carry += __shfl(x, kWave - 1);
        }
        if (lane == 0) g_vcum[nv] = carry;
    } else if (w == 0) {
        for (int b = tid - kWave; b < p.B; b += NT - kWave) {
            // nodes before b in its group, the group's first row block (see
            // shared_unit), shared tiles, node count
            const int s = g_group[b], n0 = s < kMaxGroups ? g_ncum[g_gstart[s]] : 0;
            reinterpret_cast<i32x4 *>(p.ws_seq)[b] =
                i32x4{g_ncum[b] - n0, s < kMaxGroups ? n0 * p.G / p.rows_per_block + s : 0, shared_tiles_of(b),
                      g_ncum[b + 1] - g_ncum[b]};
        }
    }
    __syncthreads();
}

// Row (node of all sequences, per head) of node `ord` of group s.
__device__ __forceinline__ size_t group_node(int s, int ord, const SharedAttnParams &p) {
    int lo = g_gstart[s], hi = g_gstart[s + 1] - 1;
    const int o = ord + g_ncum[lo];
    while (lo < hi) {                    // the last sequence whose nodes start at or before o
        const int mid = (lo + hi + 1) >> 1;
        if (g_ncum[mid] <= o) lo = mid; else hi = mid - 1;
    }
    return (size_t)lo * p.N + (o - g_ncum[lo]);
}

// Numbers of the units in ws_unit: the sequences' own ones, then the shared ones.
// A group of R rows behind X rows of groups before it has at most
// floor((X + R) / block) - floor(X / block) + 1 row blocks, so with one more per
// group before it the blocks of all groups get numbers of their own.
__device__ __forceinline__ int own_blocks(const SharedAttnParams &p) {
    return (p.N * p.G + p.own_rows - 1) / p.own_rows;
}
__device__ __forceinline__ int own_unit(int b, int g, int rb, const SharedAttnParams &p) {
    return (b * p.Hkv + g) * own_blocks(p) + rb;
}
__device__ __forceinline__ int shared_unit_of(int block, int g, const SharedAttnParams &p) {
    return p.B * p.Hkv * own_blocks(p) + block * p.Hkv + g;
}
__device__ __forceinline__ int shared_unit(int s, int g, int rb, const SharedAttnParams &p) {
    return shared_unit_of(g_ncum[g_gstart[s]] * p.G / p.rows_per_block + s + rb, g, p);
}

}  // namespace
}  // namespace tv

#include "tree_attention_own.h"

namespace tv {
namespace {

// RT > 0: the sequences' own keys are units of at most RT x 16 rows that some of
// the workgroups take wave by wave, and the others share the groups' units; RT = 0:
// all workgroups share the units of both kinds. A share may start and end inside a
// unit; a piece of one runs as in tree_attention_kernel.
template <int D, bool SMALL, int RT>
__global__ __launch_bounds__(NT) void shared_attention_kernel(SharedAttnParams p) {
    using Gm = Geo<D>;
    using Issue = TileIssue<D, NW, SMALL>;
    constexpr int NKS = D / 16;
    constexpr int NDT = D / 32;
    constexpr int LPT = Issue::kLoadsPerWave;

    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    const int wave_u = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5;
    const int col = lane & 31;
    int w = xcd_contiguous_id(blockIdx.x, p.num_wg);

    build_shared_tables<RT ? D : 0>(p, w);

    int num_wg = p.num_wg;
    int total = g_vcum[p.groups + p.B];
    if constexpr (RT > 0) {
        // Workgroups are divided by the work of the two kinds, in multiples of the XCDs
        const int shared = g_vcum[p.groups], own = total - shared;
        const int eighths = num_wg / kNumXcd;
        int ns = 0;
        if (shared > 0) {
            const long long a = (long long)shared * shared_tile_cost<D, RT>(), both = a + own;
            ns = min(max((int)((a * eighths + both / 2) / both), 1), eighths - 1) * kNumXcd;
        }
        if ((int)blockIdx.x >= ns) {
            const int o = xcd_contiguous_id(blockIdx.x - ns, num_wg - ns);
            own_shares<D, RT>(p, o * NW + wave_u, (num_wg - ns) * NW);
            w = ns + o;
            total = 0;
        } else {
            w = xcd_contiguous_id(blockIdx.x, ns);
            total = shared;
        }
        num_wg = ns;
    }
    // Workgroup u < nw takes virtual tiles [share_start(u), share_start(u + 1)):
    // shares differ by at most one tile and none is empty (nw <= total), so the
    // pieces of a split unit sit in consecutive workgroups.
    const int nw = min(num_wg, total);
    auto share_start = [&](int u) { return (int)(((long long)min(u, nw) * total) / max(nw, 1)); };
    const int start = share_start(w), end = share_start(w + 1);
    const unsigned ring_base = lds_addr(g_ring);
    Issue ld;
    ld.init(wave_u, lane, p);

    // lane-constant parts of the LDS fragment addresses (see swz)
    const unsigned k_lane = col * Gm::kRowBytes + ((half ^ swz<Gm::kChunks>(col % Gm::kChunks)) << 4);
    const int va = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const int vb = half * 4 + ((lane & 15) >> 2);
    const unsigned v_lane = vb * Gm::kRowBytes + ((va ^ swz<Gm::kChunks>(vb)) << 4) + (lane & 1) * 8;

    int pos = start;
    int anc_b = -1;                 // sequence whose ancestor sets are in g_anc
    while (pos < end) {
        // ---- locate the unit holding tile `pos`
        int lo = 0, hi = p.groups + p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (g_vcum[mid] <= pos) lo = mid; else hi = mid - 1;
        }
        int b, L, nodes, rows_b, ntp;   // rows_b: query rows per KV head of the group or sequence
        int ts = 0;                     // the unit's first tile (behind the tiles taken together)
        int sg = -1;                    // shared unit: its group; b is then the sequence whose pages are read
        const int C = p.setup_tiles;
        int off = pos - g_vcum[lo], g, rb = 0, ulen;     // ulen: real tiles of the unit
        if (RT > 0 || lo < p.groups) {
            sg = lo;
            b = g_first[sg];
            ntp = g_gtiles[sg];
            L = ntp * KT;
            nodes = 1;              // of sequence b: it has one at least
            rows_b = group_rows(sg, p);
            ulen = ntp;
            const int u = off / (C + ulen), rbs = row_blocks_of(rows_b, p);
            off -= u * (C + ulen);
            g = u / rbs;
            rb = u - g * rbs;
        } else {
            b = lo - p.groups;
            L = g_slen[b];
            nodes = g_ncum[b + 1] - g_ncum[b];
            rows_b = nodes * p.G;
            ntp = (L + KT - 1) / KT;
            ts = shared_tiles_of(b);
            const int per_g = tiles_per_head(ntp - ts, rows_b, p);
            g = off / per_g;
            off -= g * per_g;
            ulen = ntp - ts + tree_tiles_of_block(0, rows_b, p);
            while (off >= C + ulen) {
                off -= C + ulen;
                ++rb;
                ulen = ntp - ts + tree_tiles_of_block(rb, rows_b, p);
            }
        }
        // this share covers virtual tiles [off, v_end) of the unit; its real tile
        // ts + r is virtual tile C + r
        const int v_end = min(C + ulen, off + (end - pos));
        const int unit_real_start = pos - off + C;    // share coordinate of the first real tile
        const int t0 = ts + max(off - C, 0);
        pos += v_end - off;
        const int t_end = ts + v_end - C;
        if (t_end <= t0) continue;                    // only set-up tiles of this unit
        const bool complete = (t0 == ts && t_end == ts + ulen);

        // Parent links for the ancestor sets (trees of up to 64 nodes), loaded
        // before any other load of the piece so that waiting for them never
        // waits for the tile loads behind them; then the first four tiles' page ids.
        const bool need_anc = t_end > ntp && anc_b != b;
        int par_pre = -1;
        if (need_anc && wave_u == 0 && p.N <= kWave && lane < p.N)
            par_pre = p.parent[(size_t)b * p.N + lane];
        int ids[4][LPT];
        #pragma unroll
        for (int i = 0; i < 4; ++i) ld.fetch_pages(p, b, t0 + i, wave_u, ids[i]);

        // ---- this wave's 32 query rows: Q fragments stay in registers. A row past the
        // unit's last one loads the unit's first row instead and is never stored; a wave
        // without rows loads its share of the tiles and computes nothing.
        const int row = rb * p.rows_per_block + wave_u * kRowsPerWave + col;
        const bool row_ok = row < rows_b;
        const bool idle = rb * p.rows_per_block + wave_u * kRowsPerWave >= rows_b;
        const int qrow = row_ok ? row : rb * p.rows_per_block;
        const int node = sg >= 0 ? 0 : qrow / p.G;       // whose ancestors the row sees
        const int hq = g * p.G + qrow % p.G;
        const int qnode = sg >= 0 ? (int)group_node(sg, qrow / p.G, p) : b * p.N + node;   // of all sequences'
        WaveState<D> st;
        const uint16_t *qp = p.q + ((size_t)qnode * p.Hq + hq) * D + half * 8;
        #pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
            st.qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8 *>(qp + ks * 16));
        #pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
            #pragma unroll
            for (int r = 0; r < 16; ++r) st.o[dt][r] = 0.f;
        st.m_run = kNegInf;
        st.msc = 0.f;
        st.l_run = 0.f;

        const int npages = (L + p.P - 1) >> p.p_shift;
        auto kaddr_of = [&](int t) { return ring_base + (t & (NS - 1)) * Gm::kStageBytes + k_lane; };
        auto vaddr_of = [&](int t) {
            return ring_base + (t & (NS - 1)) * Gm::kStageBytes + Gm::kTileBytes + v_lane;
        };
        f32x16 s0, s1;                    // scores of the current tile: half 0, half 1

        // The piece runs in sub-ranges whose prefix pages fit the LDS page-id window
        // (one sub-range unless it spans more than kPageCache pages shorter than a load).
        for (int ta = t0; ta < t_end;) {
            const int page_first = (ta * KT) >> p.p_shift;
            int tb = t_end;
            if (ta < ntp) {
                const int t_cov = ((page_first + kPageCache) << p.p_shift) / KT;   // first tile not covered
                if (t_cov < ntp) tb = min(tb, t_cov);
            }
            if (SMALL && ta < ntp) load_pages<NT>(p, b, page_first, npages);

            // Period j computes S with K_j and PV with V_{j-1} of the sub-range's tiles and
            // issues K_{j+3} and V_{j+2} into the halves last read in period j - 1.
            const int T = tb - ta;
            int pk[LPT];                       // page ids of the next K tile to be loaded
            typename Issue::Blocks bk;         // block addresses of the last K tile issued,
            bool fast = false;                 // or, when `fast`, its common-case offset
            unsigned long long foff = 0;
            auto take_ids = [&](const int (&from)[LPT]) {
                #pragma unroll
                for (int k = 0; k < LPT; ++k) pk[k] = from[k];
            };
            auto blocks_of = [&](int i) { return ld.blocks(p, ta + i, wave_u, pk); };
            auto issue_half = [&](int i, bool is_v, const typename Issue::Blocks &bl) {
                const int t = ta + i;
                if (SMALL && t < ntp) ld.issue_small(p, t, is_v, page_first, wave_u);
                else ld.issue(bl, is_v, t & (NS - 1), wave_u);
            };
            ld.set_unit(p, b, g, L, ntp, nodes);
            // issue order K_0, V_0, K_1, V_1, K_2 (the waits below count on it)
            typename Issue::Blocks b0, b1;
            take_ids(ids[0]);
            b0 = blocks_of(0);
            if (T > 1) {
                take_ids(ids[1]);
                b1 = blocks_of(1);
            }
            if (T > 2) {
                take_ids(ids[2]);
                bk = blocks_of(2);             // K_2 now, V_2 in period 0
            }
            issue_half(0, false, b0);
            issue_half(0, true, b0);
            if (T > 1) {
                issue_half(1, false, b1);
                issue_half(1, true, b1);
            }
            if (T > 2) issue_half(2, false, bk);
            take_ids(ids[3]);
            // Ancestor sets, while the first loads are in flight, by one wave (the
            // others read them only after the next workgroup barrier).
            if (ta == t0 && need_anc) {
                if (wave_u == 0) {
                    tie(par_pre);              // first use here, behind the tile loads
                    if (p.N <= kWave) build_ancestor_masks_wave(p, par_pre);
                    else build_ancestor_masks_wave_lds(p, b);
                }
                anc_b = b;
            }

            // Loads this wave issues at the end of period i (V_{i+2}, K_{i+3} when they exist).
            auto loads_in = [&](int i) { return (i + 3 < T ? LPT : 0) + (i + 2 < T ? LPT : 0); };
            // Opening of period j: K_j and V_{j-1} have landed for every wave and every
            // wave is done with period j - 1; then tile j's mask.
            TileMask mk;
            auto open_period = [&](int j) {
                int newer;                     // loads issued after the last one period j needs
                if (j == 0) newer = LPT * ((T > 1 ? 2 : 0) + (T > 2 ? 1 : 0)) + LPT;   // V_0, K_1, V_1, K_2
                else if (j == 1) newer = LPT * ((T > 1 ? 1 : 0) + (T > 2 ? 1 : 0)) + loads_in(0);
                else if (j == 2) newer = loads_in(0) + loads_in(1);
                else newer = loads_in(j - 2) + loads_in(j - 1);
                wait_vm_at_most(newer);
                lds_barrier();
                const int t = ta + j;
                unsigned long long vis;
                if (t < ntp) {
                    const int lim_t = L - t * KT;      // keys at or past it lie beyond the prefix
                    mk.masked = lim_t < KT;
                    vis = lim_t >= KT ? ~0ull : ((1ull << lim_t) - 1ull);
                } else {
                    mk.masked = true;
                    vis = g_anc[node][t - ntp];
                }
                vis >>= half * 4;
                mk.vis_lo = (unsigned)vis;
                mk.vis_hi = (unsigned)(vis >> 32);
            };
            // End of period j: this wave's loads of K_{j+3} and V_{j+2} in one burst, then
            // the page ids of K_{j+4} by scalar loads that complete by the next barrier.
            auto close_period = [&](int j) {
                if (j + 2 < T) {                   // V_{j+2}: the addresses of K_{j+2}
                    if (fast) ld.issue_fast(foff, true, (ta + j + 2) & (NS - 1), wave_u);
                    else issue_half(j + 2, true, bk);
                }
                if (j + 3 < T) {
                    fast = !SMALL && ld.fast_offset(p, ta + j + 3, wave_u, pk[0], foff);
                    if (fast) {
                        ld.issue_fast(foff, false, (ta + j + 3) & (NS - 1), wave_u);
                    } else {
                        if (!(SMALL && ta + j + 3 < ntp)) bk = blocks_of(j + 3);
                        issue_half(j + 3, false, bk);
                    }
                }
                ld.fetch_pages(p, b, ta + j + 4, wave_u, pk);
            };
            int j = 0;
            auto run = [&](auto prev, auto cur) {
                constexpr bool P_ = decltype(prev)::value, C_ = decltype(cur)::value;
                const int jj = j;
                if (!idle)
                    tile_period<D, P_, C_>(st, s0, s1, C_ ? kaddr_of(ta + jj) : 0u,
                                           P_ ? vaddr_of(ta + jj - 1) : 0u, mk, p.scale_log2);
                if (C_) close_period(jj);
            };
            using T_ = std::true_type;
            using F_ = std::false_type;
            open_period(0);
            run(F_{}, T_{});
            for (j = 1; j < T; ++j) {
                open_period(j);
                run(T_{}, T_{});
            }
            wait_vm_at_most(0);            // V of the last tile has landed for every wave
            lds_barrier();
            run(T_{}, F_{});               // PV of the last tile
            ta = tb;
            if (ta < t_end) {
                #pragma unroll
                for (int i = 0; i < 4; ++i) ld.fetch_pages(p, b, ta + i, wave_u, ids[i]);
            }
            __syncthreads();               // ring and page ids are reused next
        }

        // ---- finish the piece
        // The normalised rows leave through this wave's slice of the (now idle) LDS ring,
        // transposed there so that every global store writes whole rows. Rows of a whole
        // unit without shared keys beside it are the result; others are parts (fp16), of a
        // whole unit in ws_whole, of a piece in a slot: slot 0 holds the piece that
        // continues a unit from before this share, slot 1 the one that starts inside it.
        const int slot = w * 2 + (unit_real_start <= start ? 0 : 1);
        const bool last = complete && sg < 0 && ts == 0;
        if (tid == 0) {
            // where the joining kernel finds the unit: the slot of its first piece
            // (-1: a whole unit) and the workgroup of its last
            int32_t *rec = p.ws_unit + 2 * (sg >= 0 ? shared_unit(sg, g, rb, p) : own_unit(b, g, rb, p));
            if (t0 == ts) rec[0] = complete ? -1 : slot;
            if (t_end == ts + ulen) rec[1] = w;
        }
        const float l_tot = halves_sum(st.l_run);
        const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
        constexpr int kPitch = D * 2 + 16;                   // LDS bytes per row (padded)
        constexpr int kRowChunks = D / 8;                     // 16-byte chunks per row
        constexpr int kRowsPerPass = kWave / kRowChunks;
        unsigned char *wbuf = g_ring + wave_u * kRowsPerWave * kPitch;
        float unscale = 1.f, scaled = inv;
        if (!last) {
            const float top = row_top(
                [&](auto take) {
                    #pragma unroll
                    for (int dt = 0; dt < NDT; ++dt)
                        #pragma unroll
                        for (int r = 0; r < 16; ++r) take(st.o[dt][r]);
                },
                halves_max);
            scaled *= part_scale(top * inv, unscale);
        }
        #pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
            #pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                bf16x4 v;
                if (last) {
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (__bf16)(st.o[dt][q4 * 4 + i] * inv);
                } else {
                    f16x4 f;
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = (_Float16)(st.o[dt][q4 * 4 + i] * scaled);
                    v = __builtin_bit_cast(bf16x4, f);
                }
                *reinterpret_cast<bf16x4 *>(wbuf + col * kPitch + (dt * 32 + q4 * 8 + half * 4) * 2) = v;
            }
        const size_t all = (size_t)p.B * p.N * p.Hq;
        #pragma unroll
        for (int k = 0; k < kRowsPerWave / kRowsPerPass; ++k) {
            const int r = k * kRowsPerPass + lane / kRowChunks, ch = lane % kRowChunks;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(wbuf + r * kPitch + ch * 16);
            const int rl = wave_u * kRowsPerWave + r;           // row within the unit's block
            if (complete) {
                const int ur = rb * p.rows_per_block + rl;
                if (ur < rows_b) {
                    const int nd = ur / p.G, h = g * p.G + ur % p.G;
                    const size_t on = sg >= 0 ? group_node(sg, nd, p) : (size_t)b * p.N + nd;
                    uint16_t *o = last ? p.out : p.ws_whole + (sg >= 0 ? 0 : all * D);
                    *reinterpret_cast<u32x4 *>(o + (on * p.Hq + h) * D + ch * 8) = v;
                }
            } else {
                *reinterpret_cast<u32x4 *>(p.ws_o + ((size_t)slot * p.rows_per_block + rl) * D + ch * 8) = v;
            }
        }
        if (half == 0) {
            const float m2 = (st.m_run == kNegInf) ? kNegInf : st.m_run * p.scale_log2;
            const f32x4 desc = {m2, l_tot, unscale, 0.f};
            const size_t at = (size_t)qnode * p.Hq + hq;
            if (!complete) p.ws_piece[(size_t)slot * p.rows_per_block + wave_u * kRowsPerWave + col] = desc;
            else if (row_ok && !last) p.ws_row[(sg >= 0 ? 0 : all) + at] = desc;
            else if (row_ok && p.lse) p.lse[at] = (m2 + __builtin_amdgcn_logf(l_tot)) * kLn2;
        }
        __syncthreads();                   // the ring is refilled by the next piece
    }

    // Rows of padding nodes (at or past a sequence's node count) are not part
    // of any unit: write them as zeros with lse -inf, a few nodes per workgroup.
    if (p.num_nodes) {
        const int chunks = p.Hq * D / 8;             // 16-byte chunks of one node's output
        for (int idx = w; idx < p.B * p.N; idx += p.num_wg) {
            const int b = idx / p.N, i = idx - b * p.N;
            if (i < g_ncum[b + 1] - g_ncum[b]) continue;
            u16x8 *op = reinterpret_cast<u16x8 *>(p.out + ((size_t)b * p.N + i) * p.Hq * D);
            for (int c = tid; c < chunks; c += NT) op[c] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (p.lse)
                for (int h = tid; h < p.Hq; h += NT) p.lse[((size_t)b * p.N + i) * p.Hq + h] = kNegInf;
        }
    }
}
// Join the results of every row of a batch with shared prefixes: those of its
// group's shared keys, if any, and those of its sequence's own keys, each one
// row or the pieces of a split unit. One thread per (row, 8 head-dim lanes), in
// the order of `out`; pieces are combined in workgroup order with an online
// log-sum-exp rescale. Rows with one whole result have it in `out` already.
template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedAttnParams p) {
    constexpr int D8 = D / 8;
    const size_t row = (size_t)blockIdx.x * (256 / D8) + threadIdx.x / D8;
    const int d8 = threadIdx.x % D8;
    const size_t rows = (size_t)p.B * p.N * p.Hq;
    if (row >= rows) return;
    const int h = (int)(row % p.Hq), i = (int)(row / p.Hq % p.N), b = (int)(row / ((size_t)p.Hq * p.N));
    const int g = h / p.G;
    const int own_row = i * p.G + h % p.G;
    // what does not depend on one another is asked for together, used or not: the
    // sequence's place, the own unit's record, and its row if it is whole
    const i32x4 sq = reinterpret_cast<const i32x4 *>(p.ws_seq)[b];
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 own = *reinterpret_cast<const i32x2 *>(
        p.ws_unit + 2 * own_unit(b, g, own_row / p.own_rows, p));
    const f16x8 own_o = *reinterpret_cast<const f16x8 *>(p.ws_whole + (rows + row) * D + d8 * 8);
    const f32x4 own_m = p.ws_row[rows + row];
    if (i >= sq[3]) return;                         // padding: written by the main kernel
    const bool shared = sq[2] > 0;
    const int group_row = sq[0] * p.G + own_row;
    if (!shared && own[0] < 0) return;
    i32x2 shr = {-1, -1};
    if (shared)
        shr = *reinterpret_cast<const i32x2 *>(
            p.ws_unit + 2 * shared_unit_of(sq[1] + group_row / p.rows_per_block, g, p));

    float M = kNegInf, den = 0.f;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // a part with maximum m[0], sum m[1] and fp16 values times m[2]
    auto add = [&](const f16x8 &v, const f32x4 &m) {
        const float Mn = fmaxf(M, m[0]);
        const float sc = (M == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
        const float wt = (m[0] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(m[0] - Mn) * m[1];
        den = den * sc + wt;
        #pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = acc[e] * sc + wt * ((float)v[e] * m[2]);
        M = Mn;
    };
    auto add_pieces = [&](int first, int last, int rl, int slot_rows, const uint16_t *o, const f32x4 *m) {
        #pragma unroll 4
        for (int u = first >> 1; u <= last; ++u) {
            // the first piece may sit in slot 1 of its workgroup; later ones start a share
            const size_t r = (size_t)(u == (first >> 1) ? first : u * 2) * slot_rows + rl;
            add(*reinterpret_cast<const f16x8 *>(o + r * D + d8 * 8), m[r]);
        }
    };
    if (own[0] < 0) add(own_o, own_m);
    else add_pieces(own[0], own[1], own_row % p.own_rows, p.own_rows, p.own_o, p.own_piece);
    if (shared && shr[0] < 0)
        add(*reinterpret_cast<const f16x8 *>(p.ws_whole + row * D + d8 * 8), p.ws_row[row]);
    else if (shared)
        add_pieces(shr[0], shr[1], group_row % p.rows_per_block, p.rows_per_block, p.ws_o, p.ws_piece);
    const float inv = den > 0.f ? 1.f / den : 0.f;
    bf16x8 o;
    #pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x8 *>(p.out + row * D + d8 * 8) = o;
    if (p.lse && d8 == 0) p.lse[row] = (M + __builtin_amdgcn_logf(den)) * kLn2;
}

template <int D, int RT>
hipError_t launch_rt(const SharedAttnParams &p, hipStream_t s) {
    return launch_kernel(p.small_pages ? shared_attention_kernel<D, true, RT> : shared_attention_kernel<D, false, RT>,
                         dim3(p.num_wg), dim3(NT), s, p);
}

template <int D>
hipError_t launch_d(const SharedAttnParams &p, hipStream_t s) {
    const hipError_t e = p.own_tiles16 == 1   ? launch_rt<D, 1>(p, s)
                         : p.own_tiles16 == 2 ? launch_rt<D, 2>(p, s)
                         : p.own_tiles16 == 3 ? launch_rt<D, 3>(p, s)
                                              : launch_rt<D, 0>(p, s);
    if (e != hipSuccess) return e;
    const size_t rows = (size_t)p.B * p.N * p.Hq, per = 256 / (D / 8);
    return launch_kernel(shared_join_kernel<D>, dim3((unsigned)((rows + per - 1) / per)), dim3(256), s, p);
}

}  // namespace

hipError_t launch_shared_attention(const SharedAttnParams &p, int head_dim, hipStream_t s) {
    return head_dim == 64 ? launch_d<64>(p, s) : launch_d<128>(p, s);
}

}  // namespace tv
