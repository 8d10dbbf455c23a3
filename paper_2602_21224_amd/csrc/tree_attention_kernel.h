// The kernels of the tree attention over a bf16 cache, and those that join a split unit's
// pieces. (tree_attention.hip explains the design; tree_attention_window.hip has the
// instances inside a window.)
#pragma once

#include "tree_attention_common.h"

namespace tv {
namespace {

// FINE: pieces of split units are fp16 times a power of two per row, with (max, sum,
// that factor's inverse, -) beside them, instead of bf16 with (max, sum): what
// tree_verify_attention_shared asks for, whose other paths keep their parts so.
// WIN: inside a window (p.window, p.sinks). A unit's prefix tiles are then those that hold
// a key which some node sees: the first ns (sinks) and those from ns + gap on. Tiles are
// counted without the gap (ntp of them) and located with it (real()); the window's edge
// depends on a node's depth, which is the size of its ancestor set less one, so pieces with
// an edge tile need those sets too.
template <int D, int NW, bool SMALL, bool NARROW, bool WHOLE, bool FINE = false, bool WIN = false>
__global__ __launch_bounds__(NW * kWave) void tree_attention_kernel(
    std::conditional_t<WIN, WindowAttnParams, AttnParams> p) {
    using Gm = Geo<D>;
    using Issue = TileIssue<D, NW, SMALL, WIN>;
    constexpr int NT = NW * kWave;
    constexpr int NKS = D / 16;
    constexpr int NDT = D / 32;
    constexpr int LPT = Issue::kLoadsPerWave;

    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    const int wave_u = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5;
    const int col = lane & 31;
    const int w = xcd_contiguous_id(blockIdx.x, p.num_wg);

    build_cumulative(p, [&](int L, int nodes) { return tiles_of_sequence(L, nodes, p); });

    const int total = g_cum[p.B];
    // Workgroup u < nw takes virtual tiles [share_start(u), share_start(u + 1)):
    // shares differ by at most one tile and none is empty (nw <= total), so the
    // pieces of a split unit sit in consecutive workgroups. Workgroups past nw
    // (only when the length hint overstated the work) have nothing to do.
    const int nw = min(p.num_wg, total);
    auto share_start = [&](int u) { return (int)(((long long)min(u, nw) * total) / max(nw, 1)); };
    auto share_of = [&](int t) { return (int)(((long long)(t + 1) * nw - 1) / total); };
    int start = share_start(w), end = share_start(w + 1);
    if constexpr (WHOLE) {
        // workgroup w takes unit w whole (unit order: sequence, KV head, row
        // block; a sequence with fewer row blocks leaves workgroups idle)
        const int rbs = row_blocks_of(p.N * p.G, p);
        const int wb = w / (p.Hkv * rbs), wg = w / rbs % p.Hkv, wr = w % rbs;
        const int rows = g_nn[wb] * p.G, ntp = (g_len[wb] + KT - 1) / KT - span_of(g_len[wb], p).gap;
        start = g_cum[wb] + wg * tiles_per_head(ntp, rows, p);
        for (int x = 0; x < min(wr, row_blocks_of(rows, p)); ++x)
            start += p.setup_tiles + ntp + tree_tiles_of_block(x, rows, p);
        end = wr < row_blocks_of(rows, p) ? start + p.setup_tiles + ntp + tree_tiles_of_block(wr, rows, p) : start;
    }
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
    if (start >= end && tid == 0) p.ws_desc[w * 4] = -1;
    while (pos < end) {
        // ---- locate the unit holding tile `pos`
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (g_cum[mid] <= pos) lo = mid; else hi = mid - 1;
        }
        const int b = lo;
        const int L = g_len[b];
        const int nodes = g_nn[b];
        const int rows_b = nodes * p.G;                 // this sequence's query rows per KV head
        const Span sp = span_of(L, p);
        const int ntp = (L + KT - 1) / KT - sp.gap;
        auto real = [&](int t) { return WIN && t >= sp.ns ? t + sp.gap : t; };
        const int C = p.setup_tiles;
        const int per_g = tiles_per_head(ntp, rows_b, p);
        int off = pos - g_cum[b];
        const int g = off / per_g;
        off -= g * per_g;
        int rb = 0;
        int ulen = ntp + tree_tiles_of_block(0, rows_b, p);     // real tiles of the unit
        while (off >= C + ulen) {
            off -= C + ulen;
            ++rb;
            ulen = ntp + tree_tiles_of_block(rb, rows_b, p);
        }
        // this share covers virtual tiles [off, v_end) of the unit; real tile
        // r is virtual tile C + r
        const int v_end = min(C + ulen, off + (end - pos));
        const int unit_real_start = pos - off + C;    // share coordinate of real tile 0
        const int t0 = max(off - C, 0);
        // Page ids of the first four tiles (scalar loads): for narrow units first
        // of all, so that their latency overlaps the rest of the set-up; for the
        // others after the parent links (holding them that long costs the
        // eight-wave kernel spills). Later sub-ranges fetch their own.
        int ids[4][Issue::kLoadsPerWave];
        if constexpr (NARROW) {
            #pragma unroll
            for (int i = 0; i < 4; ++i) ld.fetch_pages(p, b, real(t0 + i), wave_u, ids[i]);
        }
        if (pos == start && tid == 0) {
            // the merge kernel's entry for this workgroup: the split unit whose
            // last piece is this share's first, if any
            const int wf = share_of(unit_real_start);
            const bool mine = unit_real_start < start && share_of(unit_real_start + ulen - 1) == w;
            *reinterpret_cast<i32x4 *>(p.ws_desc + w * 4) =
                mine ? i32x4{b, g, rb | (nodes << 8), wf * 2 + (unit_real_start <= share_start(wf) ? 0 : 1)}
                     : i32x4{-1, 0, 0, 0};
        }
        pos += v_end - off;
        const int t_end = v_end - C;
        if (t_end <= t0) continue;                    // only set-up tiles of this unit
        const bool complete = (t0 == 0 && t_end == ulen);

        // Parent links for the ancestor sets (trees of up to 64 nodes), loaded
        // before any other load of the piece so that waiting for them never
        // waits for the tile loads behind them.
        const bool has_tree = t_end > ntp;
        const bool edge = WIN && t_end > sp.ns && real(max(t0, sp.ns)) * KT < sp.lo0 + p.N - 1;
        const bool need_anc = (has_tree || edge) && anc_b != b;
        int par_pre = -1;
        if (need_anc && wave_u == 0 && p.N <= kWave && lane < p.N)
            par_pre = p.parent[(size_t)b * p.N + lane];
        if constexpr (!NARROW) {
            #pragma unroll
            for (int i = 0; i < 4; ++i) ld.fetch_pages(p, b, real(t0 + i), wave_u, ids[i]);
        }

        // ---- this wave's 32 query rows: Q fragments stay in registers. A row
        // past the unit's last one loads the unit's first row instead (rows are
        // independent through both products and the softmax, and such rows are
        // never stored), so the loads need no branch and nothing waits for them
        // before the first score product.
        const int row = rb * p.rows_per_block + wave_u * kRowsPerWave + col;
        const bool row_ok = row < rows_b;
        const int qrow = row_ok ? row : rb * p.rows_per_block;
        const int node = qrow / p.G;
        const int hq = g * p.G + qrow % p.G;
        WaveState<D> st;
        NarrowState<D> ns;
        // narrow units: lane l holds row l % 16 (rows past the unit's last load
        // its first row, never stored) and head-dim columns 8 (l / 16) + 32 ks
        const int nrow = NARROW ? min(lane & 15, rows_b - 1) : 0;
        const int nnode = nrow / p.G;
        if constexpr (!NARROW) {
            const uint16_t *qp = p.q + (((size_t)b * p.N + node) * p.Hq + hq) * D + half * 8;
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
        } else {
            const int nhq = g * p.G + nrow % p.G;
            const uint16_t *qp = p.q + (((size_t)b * p.N + nnode) * p.Hq + nhq) * D + (lane >> 4) * 8;
            #pragma unroll
            for (int ks = 0; ks < D / 32; ++ks)
                ns.qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8 *>(qp + ks * 32));
            #pragma unroll
            for (int db = 0; db < D / 16; ++db) ns.o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
            ns.m_run = kNegInf;
            ns.msc = 0.f;
            ns.l_run = 0.f;
        }

        const int npages = (L + p.P - 1) >> p.p_shift;
        auto kaddr_of = [&](int t) { return ring_base + (t & (NS - 1)) * Gm::kStageBytes + k_lane; };
        auto vaddr_of = [&](int t) {
            return ring_base + (t & (NS - 1)) * Gm::kStageBytes + Gm::kTileBytes + v_lane;
        };
        // Scores of the current tile: half 0 in s0, half 1 in s1 (exponentiated
        // early in the next period).
        f32x16 s0, s1;

        // The segment runs in sub-ranges whose prefix pages fit the LDS page-id
        // window (one sub-range unless a piece spans more than kPageCache pages).
        for (int ta = t0; ta < t_end;) {
            const int page_first = (real(ta) * KT) >> p.p_shift;
            int tb = t_end;
            if (ta < ntp) {
                // first tile not covered
                const int t_cov = page_window_end(page_first, p.p_shift) - (WIN && ta >= sp.ns ? sp.gap : 0);
                if (t_cov < ntp) tb = min(tb, t_cov);
                if (WIN && SMALL && ta < sp.ns && sp.gap > 0) tb = min(tb, sp.ns);
            }
            const bool first = (ta == t0);
            // page ids in LDS only for pages shorter than a load block; ancestor
            // sets only when this piece reaches the tree tiles and the workgroup
            // has not built them for this sequence already
            const bool want_anc = first && need_anc;
            if (SMALL && ta < ntp) load_pages<NT>(p, b, page_first, npages);

            const int T = tb - ta;
            // Tile i of the sub-range (K and V of tile ta + i) goes to ring stage
            // (ta + i) % NS. Period j computes S with K_j and PV with V_{j-1}, and
            // issues K_{j+3} and V_{j+2}: the K half it refills last held K_{j-1}
            // (read in period j - 1), the V half V_{j-2} (read in period j - 1),
            // both before the barrier that opens period j. Every load is issued
            // about three periods before it is read.
            int pk[LPT];                       // page ids of the next K tile to be loaded
            typename Issue::Blocks bk;         // block addresses of the last K tile issued,
            bool fast = false;                 // or, when `fast`, its common-case offset
            unsigned long long foff = 0;
            auto blocks_of = [&](int i) { return ld.blocks(p, real(ta + i), wave_u, pk); };
            auto issue_half = [&](int i, bool is_v, const typename Issue::Blocks &bl) {
                const int t = ta + i;
                if (SMALL && t < ntp) ld.issue_small(p, real(t), is_v, page_first, wave_u, t & (NS - 1));
                else ld.issue(bl, is_v, t & (NS - 1), wave_u);
            };
            ld.set_unit(p, b, g, L, ntp + sp.gap, nodes);
            if constexpr (WIN) {
                ld.lo = sp.lo;
                ld.sink_end = sp.sinks;
            }
            {
                // narrow units: full prefix tiles take the fast address path here too
                typename Issue::Blocks b0, b1;
                unsigned long long f0 = 0, f1 = 0;
                const bool fa0 = NARROW && !SMALL && ld.fast_offset(p, real(ta), wave_u, ids[0][0], f0);
                const bool fa1 = NARROW && !SMALL && T > 1 && ld.fast_offset(p, real(ta + 1), wave_u, ids[1][0], f1);
                fast = NARROW && !SMALL && T > 2 && ld.fast_offset(p, real(ta + 2), wave_u, ids[2][0], foff);
                if (!fa0) {
                    #pragma unroll
                    for (int k = 0; k < LPT; ++k) pk[k] = ids[0][k];
                    b0 = blocks_of(0);
                }
                if (T > 1 && !fa1) {
                    #pragma unroll
                    for (int k = 0; k < LPT; ++k) pk[k] = ids[1][k];
                    b1 = blocks_of(1);
                }
                if (T > 2 && !fast) {
                    #pragma unroll
                    for (int k = 0; k < LPT; ++k) pk[k] = ids[2][k];
                    bk = blocks_of(2);         // K_2 now, V_2 in period 0 (narrow: now)
                }
                auto issue_pro = [&](int i, bool is_v, bool fa, unsigned long long fo,
                                     const typename Issue::Blocks &bl) {
                    if (fa) ld.issue_fast(fo, is_v, (ta + i) & (NS - 1), wave_u);
                    else issue_half(i, is_v, bl);
                };
                // issue order K_0, V_0, K_1, V_1, K_2 (, V_2) (the waits below count on it)
                issue_pro(0, false, fa0, f0, b0);
                issue_pro(0, true, fa0, f0, b0);
                if (T > 1) {
                    issue_pro(1, false, fa1, f1, b1);
                    issue_pro(1, true, fa1, f1, b1);
                }
                if (T > 2) issue_pro(2, false, fast, foff, bk);
                if (NARROW && T > 2) issue_pro(2, true, fast, foff, bk);
                #pragma unroll
                for (int k = 0; k < LPT; ++k) pk[k] = ids[3][k];
            }
            // Ancestor sets, while the first loads are in flight, by one wave (the
            // others read them only after the next workgroup barrier): in
            // registers up to 64 nodes, else in LDS.
            if (want_anc) {
                if (wave_u == 0) {
                    tie(par_pre);              // first use here, behind the tile loads
                    if (p.N <= kWave) build_ancestor_masks_wave(p, par_pre);
                    else build_ancestor_masks_wave_lds(p, b);
                }
                anc_b = b;
            }

            // Loads this wave issues at the end of period i (V_{i+2}, K_{i+3} when they exist).
            auto loads_in = [&](int i) { return (i + 3 < T ? LPT : 0) + (i + 2 < T ? LPT : 0); };
            // Opening of period j: K_j and V_{j-1} have landed for every wave (this
            // wave's later loads may still be in flight) and every wave is done
            // with period j - 1; then tile j's mask.
            TileMask mk;
            unsigned long long nvis = ~0ull;   // narrow units: the visible keys of the lane's row
            auto open_period = [&](int j) {
                int newer;                     // loads issued after the last one period j needs
                if (NARROW) newer = 2 * LPT * ((j + 1 < T ? 1 : 0) + (j + 2 < T ? 1 : 0));   // tiles j+1, j+2
                else if (j == 0) newer = LPT * ((T > 1 ? 2 : 0) + (T > 2 ? 1 : 0)) + LPT;   // V_0, K_1, V_1, K_2
                else if (j == 1) newer = LPT * ((T > 1 ? 1 : 0) + (T > 2 ? 1 : 0)) + loads_in(0);
                else if (j == 2) newer = loads_in(0) + loads_in(1);
                else newer = loads_in(j - 2) + loads_in(j - 1);
                wait_vm_at_most(newer);
                lds_barrier();
                const int t = ta + j;
                unsigned long long vis;
                if (t < ntp) {
                    const int base = real(t) * KT;
                    const int lim_t = L - base;        // keys at or past it lie beyond the prefix
                    mk.masked = lim_t < KT;
                    vis = lim_t >= KT ? ~0ull : ((1ull << lim_t) - 1ull);
                    if (WIN && !window_clear(sp, base, p.N)) {
                        mk.masked = true;
                        vis &= window_bits(sp, base, g_anc[NARROW ? nnode : node]);
                    }
                } else {
                    mk.masked = true;
                    vis = window_path(g_anc[NARROW ? nnode : node], t - ntp, L, p);
                }
                nvis = vis;
                vis >>= half * 4;
                mk.vis_lo = (unsigned)vis;
                mk.vis_hi = (unsigned)(vis >> 32);
            };
            // End of period j: this wave's loads of K_{j+3} and V_{j+2}, all at
            // once. (LDS-DMA writes slow down the LDS operand reads of every wave
            // of the CU; one burst per period costs far less than loads spread
            // between the MFMAs.) The K half they refill last held K_{j-1}, the V
            // half V_{j-2}, both read before the barrier that opened period j.
            // Then the page ids of K_{j+4}, by scalar loads that complete by the
            // next barrier.
            auto close_period = [&](int j) {
                if (j + 2 < T) {                   // V_{j+2}: the addresses of K_{j+2}
                    if (fast) ld.issue_fast(foff, true, (ta + j + 2) & (NS - 1), wave_u);
                    else issue_half(j + 2, true, bk);
                }
                if (j + 3 < T) {
                    fast = !SMALL && ld.fast_offset(p, real(ta + j + 3), wave_u, pk[0], foff);
                    if (fast) {
                        ld.issue_fast(foff, false, (ta + j + 3) & (NS - 1), wave_u);
                    } else {
                        if (!(SMALL && ta + j + 3 < ntp)) bk = blocks_of(j + 3);
                        issue_half(j + 3, false, bk);
                    }
                }
                ld.fetch_pages(p, b, real(ta + j + 4), wave_u, pk);
            };
            int j = 0;
            auto run = [&](auto prev, auto cur) {
                constexpr bool P_ = decltype(prev)::value, C_ = decltype(cur)::value;
                const int jj = j;
                tile_period<D, P_, C_>(st, s0, s1, C_ ? kaddr_of(ta + jj) : 0u,
                                       P_ ? vaddr_of(ta + jj - 1) : 0u, mk, p.scale_log2);
                if (C_) close_period(jj);
            };
            // Before the last PV: V of the last tile has landed for every wave.
            auto close_periods = [&]() {
                wait_vm_at_most(0);
                lds_barrier();
            };
            using T_ = std::true_type;
            using F_ = std::false_type;
            if constexpr (NARROW) {
                // tile t is computed whole by wave t % NW (= its ring stage); at
                // the end of period j every wave issues its share of tile j + 3
                // (K and V), whose stage last held tile j - 1, computed in period
                // j - 1, before the barrier that opened period j
                for (j = 0; j < T; ++j) {
                    open_period(j);
                    const int t = ta + j;
                    if ((t & (NS - 1)) == wave_u)
                        narrow_tile<D>(ns, ring_base + (t & (NS - 1)) * Gm::kStageBytes,
                                       ring_base + (t & (NS - 1)) * Gm::kStageBytes + Gm::kTileBytes,
                                       mk.masked, nvis, p.scale_log2, lane);
                    if (j + 3 < T) {
                        fast = !SMALL && ld.fast_offset(p, real(t + 3), wave_u, pk[0], foff);
                        if (fast) {
                            ld.issue_fast(foff, false, (t + 3) & (NS - 1), wave_u);
                            ld.issue_fast(foff, true, (t + 3) & (NS - 1), wave_u);
                        } else {
                            if (!(SMALL && t + 3 < ntp)) bk = blocks_of(j + 3);
                            issue_half(j + 3, false, bk);
                            issue_half(j + 3, true, bk);
                        }
                    }
                    ld.fetch_pages(p, b, real(t + 4), wave_u, pk);
                }
            } else {
                open_period(0);
                run(F_{}, T_{});
                for (j = 1; j < T; ++j) {
                    open_period(j);
                    run(T_{}, T_{});
                }
                close_periods();
                run(T_{}, F_{});               // PV of the last tile
            }
            ta = tb;
            if (ta < t_end) {
                #pragma unroll
                for (int i = 0; i < 4; ++i) ld.fetch_pages(p, b, real(ta + i), wave_u, ids[i]);
            }
            __syncthreads();               // ring and page ids are reused next
        }

        // ---- finish the segment
        // The normalised rows leave through this wave's slice of the (now idle)
        // LDS ring, transposed there so that every global store writes whole
        // rows (16 lanes x 16 bytes per 256-byte row) instead of 8-byte pieces
        // of 32 rows. A complete unit writes out and lse; a piece of a split
        // unit writes its output normalised by its own sum (bf16) and its (max,
        // sum) pair (fp32): slot 0 holds the piece that continues a unit from
        // before this share, slot 1 the one that starts inside it.
        const int slot = w * 2 + (unit_real_start <= start ? 0 : 1);
        if constexpr (!NARROW) {
            const float l_tot = halves_sum(st.l_run);
            const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
            constexpr int kPitch = D * 2 + 16;                   // LDS bytes per row (padded)
            constexpr int kRowChunks = D / 8;                     // 16-byte chunks per row
            constexpr int kRowsPerPass = kWave / kRowChunks;
            unsigned char *wbuf = g_ring + wave_u * kRowsPerWave * kPitch;
            [[maybe_unused]] float unscale = 1.f, scaled = inv;
            if constexpr (FINE) {
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
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (__bf16)(st.o[dt][q4 * 4 + i] * inv);
                    if constexpr (FINE) {
                        if (!complete) {
                            f16x4 f;
                            #pragma unroll
                            for (int i = 0; i < 4; ++i) f[i] = (_Float16)(st.o[dt][q4 * 4 + i] * scaled);
                            v = __builtin_bit_cast(bf16x4, f);
                        }
                    }
                    *reinterpret_cast<bf16x4 *>(wbuf + col * kPitch + (dt * 32 + q4 * 8 + half * 4) * 2) = v;
                }
            #pragma unroll
            for (int k = 0; k < kRowsPerWave / kRowsPerPass; ++k) {
                const int r = k * kRowsPerPass + lane / kRowChunks, ch = lane % kRowChunks;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(wbuf + r * kPitch + ch * 16);
                const int rl = wave_u * kRowsPerWave + r;           // row within the unit's block
                if (complete) {
                    const int ur = rb * p.rows_per_block + rl;
                    if (ur < rows_b) {
                        const int nd = ur / p.G, h = g * p.G + ur % p.G;
                        *reinterpret_cast<u32x4 *>(p.out + (((size_t)b * p.N + nd) * p.Hq + h) * D + ch * 8) = v;
                    }
                } else {
                    *reinterpret_cast<u32x4 *>(p.ws_o + ((size_t)slot * p.rows_per_block + rl) * D + ch * 8) = v;
                }
            }
            if (half == 0) {
                if (complete) {
                    if (row_ok && p.lse)
                        p.lse[((size_t)b * p.N + node) * p.Hq + hq] =
                            st.m_run * p.scale + __builtin_amdgcn_logf(l_tot) * kLn2;
                } else {
                    const int rloc = wave_u * kRowsPerWave + col;
                    float *pm = p.ws_ml + ((size_t)slot * p.rows_per_block + rloc) * (FINE ? 4 : 2);
                    pm[0] = part_max(st.m_run, l_tot, p.scale_log2);
                    pm[1] = l_tot;
                    if constexpr (FINE) pm[2] = unscale;
                }
            }
        } else {
            // Narrow units: the waves' (max, sum, O^T) of the 16 rows meet in
            // the idle ring and combine with the log-sum-exp rule; thread
            // (row, 8-column chunk) writes one 16-byte piece of the row.
            constexpr int kCh = D / 8;
            float *ow = reinterpret_cast<float *>(g_ring);                 // [NW][16][D]
            float *mlw = ow + NW * 16 * D;                                  // [NW][16][2]
            const float lw = rows_sum(ns.l_run);
            #pragma unroll
            for (int db = 0; db < D / 16; ++db)
                *reinterpret_cast<f32x4 *>(ow + ((size_t)wave_u * 16 + (lane & 15)) * D + db * 16 +
                                           4 * (lane >> 4)) = ns.o[db];
            if (lane < 16) {
                mlw[(wave_u * 16 + lane) * 2] = ns.m_run;
                mlw[(wave_u * 16 + lane) * 2 + 1] = lw;
            }
            __syncthreads();
            const int nrows = min(16, rows_b);
            const float c = p.scale_log2;
            for (int task = tid; task < 16 * kCh; task += NT) {
                const int r = task / kCh, ch = task % kCh;
                if (r >= nrows) continue;
                float M = kNegInf;
                #pragma unroll
                for (int u = 0; u < NW; ++u) M = fmaxf(M, mlw[(u * 16 + r) * 2]);
                float Lsum = 0.f;
                float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int u = 0; u < NW; ++u) {
                    const float mu = mlw[(u * 16 + r) * 2];
                    const float sc = (mu == kNegInf) ? 0.f : __builtin_amdgcn_exp2f((mu - M) * c);
                    Lsum += sc * mlw[(u * 16 + r) * 2 + 1];
                    const f32x4 a0 = *reinterpret_cast<const f32x4 *>(ow + ((size_t)u * 16 + r) * D + ch * 8);
                    const f32x4 a1 = *reinterpret_cast<const f32x4 *>(ow + ((size_t)u * 16 + r) * D + ch * 8 + 4);
                    #pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[e] += sc * a0[e];
                        acc[4 + e] += sc * a1[e];
                    }
                }
                const float inv = Lsum > 0.f ? 1.f / Lsum : 0.f;
                bf16x8 o;
                #pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (__bf16)(acc[e] * inv);
                if (complete) {
                    const int nd = r / p.G, h = g * p.G + r % p.G;
                    *reinterpret_cast<bf16x8 *>(p.out + (((size_t)b * p.N + nd) * p.Hq + h) * D + ch * 8) = o;
                    if (ch == 0 && p.lse)
                        p.lse[((size_t)b * p.N + nd) * p.Hq + h] = M * p.scale + __builtin_amdgcn_logf(Lsum) * kLn2;
                } else {
                    [[maybe_unused]] float unscale = 1.f;
                    if constexpr (FINE) {
                        const float top = row_top(
                            [&](auto take) {
                                #pragma unroll
                                for (int e = 0; e < 8; ++e) take(acc[e]);
                            },
                            [&](float x) {
                                #pragma unroll
                                for (int off = 1; off < kCh; off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
                                return x;
                            });
                        const float scaled = inv * part_scale(top * inv, unscale);
                        f16x8 f;
                        #pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = (_Float16)(acc[e] * scaled);
                        o = __builtin_bit_cast(bf16x8, f);
                    }
                    *reinterpret_cast<bf16x8 *>(p.ws_o + ((size_t)slot * p.rows_per_block + r) * D + ch * 8) = o;
                    if (ch == 0) {
                        float *pm = p.ws_ml + ((size_t)slot * p.rows_per_block + r) * (FINE ? 4 : 2);
                        pm[0] = part_max(M, Lsum, c);
                        pm[1] = Lsum;
                        if constexpr (FINE) pm[2] = unscale;
                    }
                }
            }
        }
        __syncthreads();                   // the ring is refilled by the next piece
    }

    // Rows of padding nodes (at or past a sequence's node count) are not part
    // of any unit: write them as zeros with lse -inf, a few nodes per workgroup.
    if (p.num_nodes) {
        const int chunks = p.Hq * D / 8;             // 16-byte chunks of one node's output
        for (int idx = w; idx < p.B * p.N; idx += p.num_wg) {
            const int b = idx / p.N, i = idx - b * p.N;
            if (i < g_nn[b]) continue;
            u16x8 *op = reinterpret_cast<u16x8 *>(p.out + ((size_t)b * p.N + i) * p.Hq * D);
            for (int c = tid; c < chunks; c += NT) op[c] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
            if (p.lse)
                for (int h = tid; h < p.Hq; h += NT) p.lse[((size_t)b * p.N + i) * p.Hq + h] = kNegInf;
        }
    }
}

// Merge the pieces of every split unit. Block (chunk, h) serves the workgroup
// w that ran as block h of the main kernel, so it sits on the same XCD and
// finds the newest partials in that XCD's L2. If w finished a unit that began
// in an earlier share, the block merges a chunk of that unit's rows: one
// thread per (row, 8 head-dim lanes), pieces combined in workgroup order with
// an online log-sum-exp rescale (one pass, all loads of a piece independent).
template <int D>
__global__ __launch_bounds__(256) void tree_attention_merge_kernel(AttnParams p, int stride) {
    constexpr int D8 = D / 8;
    constexpr int kRowsPerWg = 256 / D8;
    const int h = blockIdx.x % stride;
    const int rchunk = blockIdx.x / stride;
    if (h >= p.num_wg) return;
    const int w = xcd_contiguous_id(h, p.num_wg);
    const i32x4 d = ((const CONST_AS i32x4 *)p.ws_desc)[w];
    const int b = d[0];
    if (b < 0) return;
    const int g = d[1], rb = d[2] & 0xFF, s0 = d[3];
    const int rows_b = (d[2] >> 8) * p.G;
    const int wf = s0 >> 1;

    const int rl = rchunk * kRowsPerWg + threadIdx.x / D8;
    const int d8 = threadIdx.x % D8;
    const int row = rb * p.rows_per_block + rl;
    if (rl >= p.rows_per_block || row >= rows_b) return;

    float M = kNegInf, den = 0.f;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    #pragma unroll 4
    for (int u = wf; u <= w; ++u) {
        // the first piece may sit in slot 1 of its workgroup; later ones start a share
        const int slot = u == wf ? s0 : u * 2;
        const size_t r = (size_t)slot * p.rows_per_block + rl;
        const f32x2 ml = *reinterpret_cast<const f32x2 *>(p.ws_ml + r * 2);
        const bf16x8 v = *reinterpret_cast<const bf16x8 *>(p.ws_o + r * D + d8 * 8);
        const float Mn = fmaxf(M, ml[0]);
        const float sc = (M == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
        const float wt = (ml[0] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(ml[0] - Mn) * ml[1];
        den = den * sc + wt;
        #pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = acc[i] * sc + wt * (float)v[i];
        M = Mn;
    }
    const int node = row / p.G;
    const int hq = g * p.G + row % p.G;
    const float inv = den > 0.f ? 1.f / den : 0.f;
    bf16x8 o;
    #pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)(acc[i] * inv);
    *reinterpret_cast<bf16x8 *>(p.out + (((size_t)b * p.N + node) * p.Hq + hq) * D + d8 * 8) = o;
    if (p.lse && d8 == 0)
        p.lse[((size_t)b * p.N + node) * p.Hq + hq] = (M + __builtin_amdgcn_logf(den)) * kLn2;
}

// The same of fp16 pieces with four floats a row, and up to eight pieces' loads at once
// (the last one's again behind the end): with the loop above, whose loads came out one
// after the other here, two sequences x 26 nodes of head size 64 over 10000 keys took 36
// us a call, 27 so; the plain pieces 23.
template <int D>
__global__ __launch_bounds__(256) void tree_attention_merge_fine_kernel(AttnParams p, int stride) {
    constexpr int D8 = D / 8;
    constexpr int kRowsPerWg = 256 / D8;
    const int h = blockIdx.x % stride;
    const int rchunk = blockIdx.x / stride;
    if (h >= p.num_wg) return;
    const int w = xcd_contiguous_id(h, p.num_wg);
    const i32x4 d = ((const CONST_AS i32x4 *)p.ws_desc)[w];
    const int b = d[0];
    if (b < 0) return;
    const int g = d[1], rb = d[2] & 0xFF, s0 = d[3];
    const int rows_b = (d[2] >> 8) * p.G;
    const int wf = s0 >> 1;

    const int rl = rchunk * kRowsPerWg + threadIdx.x / D8;
    const int d8 = threadIdx.x % D8;
    const int row = rb * p.rows_per_block + rl;
    if (rl >= p.rows_per_block || row >= rows_b) return;

    float M = kNegInf, den = 0.f;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto add = [&](auto count, int u0) {
        constexpr int n = decltype(count)::value;
        f32x4 ml[n];
        f16x8 v[n];
        #pragma unroll
        for (int k = 0; k < n; ++k) {
            const int u = min(u0 + k, w), slot = u == wf ? s0 : u * 2;
            const size_t r = (size_t)slot * p.rows_per_block + rl;
            ml[k] = *reinterpret_cast<const f32x4 *>(p.ws_ml + r * 4);
            v[k] = *reinterpret_cast<const f16x8 *>(p.ws_o + r * D + d8 * 8);
        }
        __builtin_amdgcn_sched_barrier(0);
        #pragma unroll
        for (int k = 0; k < n; ++k) {
            if (u0 + k > w) break;                   // a repeat: left out, 0 times an infinity is NaN
            const float m = ml[k][0];
            const float Mn = fmaxf(M, m);
            const float sc = (M == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(M - Mn);
            const float wt = (m == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(m - Mn) * ml[k][1];
            den = den * sc + wt;
            #pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = acc[i] * sc + wt * ((float)v[k][i] * ml[k][2]);
            M = Mn;
        }
    };
    if (w - wf == 1) {
        add(std::integral_constant<int, 2>{}, wf);
    } else {
        for (int u = wf; u <= w; u += w - u < 4 ? 4 : 8) {
            if (w - u < 4) add(std::integral_constant<int, 4>{}, u);
            else add(std::integral_constant<int, 8>{}, u);
        }
    }
    const int node = row / p.G;
    const int hq = g * p.G + row % p.G;
    const float inv = den > 0.f ? 1.f / den : 0.f;
    bf16x8 o;
    #pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (__bf16)(acc[i] * inv);
    *reinterpret_cast<bf16x8 *>(p.out + (((size_t)b * p.N + node) * p.Hq + hq) * D + d8 * 8) = o;
    if (p.lse && d8 == 0)
        p.lse[((size_t)b * p.N + node) * p.Hq + hq] = (M + __builtin_amdgcn_logf(den)) * kLn2;
}

}  // namespace
}  // namespace tv
