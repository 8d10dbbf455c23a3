// Tree-masked attention over a prefix held in 4 bits for units of many query rows, for
// gfx950 (tree_attention_kv4.hip has those of few).
//
// A unit's row block is 128 RB rows: four waves, one per SIMD, of 32 RB rows each, which
// step through the block's 64-key tiles together, one barrier per tile. Such a call is
// bound by the matrix cores and the softmax between their instructions, not by bytes, so
// the codes are converted once per workgroup, a quarter by each wave, into bf16 tiles in
// LDS, and the products are those of the bf16 cache (v_mfma_f32_32x32x16_bf16, keys on M).
// With RB = 2 each operand read from LDS serves two products: the reads, which keep the LDS
// busy as long as the matrix cores are at 32 rows a wave, are halved.
//
// Period j of a wave (tile j of the piece):
//   part A  S_j^T = K_j Q^T; between the MFMAs the exponentials of tile j-1's second half
//           and the conversion of K_{j+1}
//   part B  O^T += V_{j-1}^T P_{j-1}^T; between them tile j's mask, maximum and running
//           maximum, the exponentials of its first half, the conversion of V_j
// K_{j+1} goes where K_{j-1} was and V_j where V_{j-2} was, both read before the barrier
// that opened the period. Codes are loaded into registers two periods ahead.
// The tree's rows are bf16 already: direct-to-LDS loads into two tiles of their own at the
// start of the piece (a third and fourth tile of a large tree: into the converted tiles'
// places once those are free).
#include "tree_attention_kv4.h"

namespace tv {
namespace {

template <int D, int RB>
struct WideState {
    bf16x8 qf[RB][D / 16];
    f32x16 o[RB][D / 32];
    u32x4 pb[RB][4];                       // P^T as bf16 pairs, 16 keys per k-step
    f32x16 s0[RB];                         // this tile's scores of keys 0 .. 31
    float m_run[RB], msc[RB], l_run[RB];
};

// A lane's share of one tile of K (or V): D/4 values of one key.
template <int D>
struct Part4 {
    unsigned x[D / 32];
    unsigned e;                            // scale byte
    unsigned keep;                         // all ones, or 0 if no node sees the key
};

template <int D>
__device__ __forceinline__ void load_part(Part4<D> &r, const Kv4AttnParams &p, long long at, bool is_v, int g) {
    const long long row = max(at, 0ll);
    load_dwords(r.x, (is_v ? p.v4 : p.k4) + row * (D / 2) + g * (D / 8));
    r.e = p.scales[row * (D / 16) + (is_v ? D / kBlock4 : 0) + (g * (D / 4)) / kBlock4];
    r.keep = at >= 0 ? ~0u : 0u;
}

// Eight of its values into the tile at `row` (the lane's key row, chunks swizzled by key).
template <int D>
__device__ __forceinline__ void convert_chunk(const Part4<D> &r, unsigned char *row, int chunk0, int key, int i) {
    constexpr int C = Geo<D>::kChunks;
    *reinterpret_cast<bf16x8 *>(row + (((chunk0 + i) ^ swz<C>(key % C)) << 4)) =
        from4x8(r.x[i] & r.keep, scale4(r.keep ? r.e : 127u));
}

// f(0), f(1), .., f(N - 1) with constants.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}

// Reads of the operands, whose waits the caller writes.
template <int OFFSET>
__device__ __forceinline__ u32x4 read_rows(unsigned addr) {
    u32x4 x;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(x) : "v"(addr), "i"(OFFSET));
    return x;
}
template <int OFFSET>
__device__ __forceinline__ u32x2 read_columns(unsigned addr) {
    u32x2 x;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(x) : "v"(addr), "i"(OFFSET));
    return x;
}

// One period. s1p: the previous tile's second half of scores, s1: this tile's. conv(i),
// i < 2 (D / 32): the conversions of K (first) and V.
template <int D, int RB, bool PREV, bool CUR, typename Conv>
__device__ __forceinline__ void wide_period(WideState<D, RB> &st, f32x16 (&s1p)[RB], f32x16 (&s1)[RB], unsigned kaddr,
                                            unsigned vaddr, const TileMask (&mk)[RB], float c, Conv conv) {
    using Gm = Geo<D>;
    constexpr int NKS = D / 16, NDT = D / 32;
    constexpr int C = Gm::kChunks;
    constexpr int SA = 2 * NKS, SB = 4 * NDT, NSLOT = SA + SB;
    constexpr int R = 2;                                   // operand reads run this many slots ahead
    constexpr int PPA = 8 / SA > 0 ? 8 / SA : 1;           // half-1 pairs per part-A slot
    constexpr int EA = 8 / PPA;                            // part-A slots with exponentials
    constexpr int B0 = NDT > 6 ? NDT : 6;                  // first part-B slot of the half-0 pairs
    constexpr int NC = D / 32;                             // conversions of K, and of V
    auto ops = [](int s) constexpr { return s < SA ? (CUR ? 1 : 0) : s < NSLOT ? (PREV ? 2 : 0) : 0; };
    u32x4 kb[SA];
    u32x2 vb[SB][2];
    auto issue_reads = [&](auto slot) __attribute__((always_inline)) {
        constexpr int s = decltype(slot)::value;
        if constexpr (s < SA && CUR) {
            constexpr int hf = s / NKS, ks = s % NKS;
            kb[s] = read_rows<hf * 32 * Gm::kRowBytes>(kaddr ^ ((unsigned)ks << 5));
        } else if constexpr (s >= SA && s < NSLOT && PREV) {
            constexpr int b = s - SA, kk = b / NDT, dt = b % NDT;
            constexpr unsigned flip0 = (unsigned)((dt * 4) ^ swz<C>(0)) << 4, flip1 = (unsigned)((dt * 4) ^ swz<C>(8 % C)) << 4;
            vb[b][0] = read_columns<kk * 16 * Gm::kRowBytes>(vaddr ^ flip0);
            vb[b][1] = read_columns<(kk * 16 + 8) * Gm::kRowBytes>(vaddr ^ flip1);
        }
    };
    float psa[RB], psb[RB], m8[RB][4], alpha[RB];
    bool any_raise[RB];
    #pragma unroll
    for (int r = 0; r < RB; ++r) {
        psa[r] = psb[r] = 0.f;
        alpha[r] = 1.f;
        any_raise[r] = false;
    }
    auto score = [&](auto hf_, int r) __attribute__((always_inline)) -> f32x16 & {
        if constexpr (decltype(hf_)::value == 0) return st.s0[r];
        else return s1[r];
    };
    each_of(issue_reads, std::make_integer_sequence<int, R>{});
    each_of([&](auto slot) __attribute__((always_inline)) {
        constexpr int s = decltype(slot)::value;
        issue_reads(std::integral_constant<int, s + R>{});
        if constexpr (s < SA && CUR) {
            constexpr int hf = s / NKS, ks = s % NKS;
            lds_wait<ops(s + 1) + ops(s + 2)>();
            tie(kb[s]);
            #pragma unroll
            for (int r = 0; r < RB; ++r) {
                f32x16 &to = score(std::integral_constant<int, hf>{}, r);
                to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kb[s]), st.qf[r][ks],
                                                             ks == 0 ? f32x16{} : to, 0, 0, 0);
            }
        }
        if constexpr (s >= SA && PREV) {
            constexpr int b = s - SA, kk = b / NDT, dt = b % NDT;
            lds_wait<ops(s + 1) + ops(s + 2)>();
            tie(vb[b][0]);
            tie(vb[b][1]);
            const u32x4 a = {vb[b][0][0], vb[b][0][1], vb[b][1][0], vb[b][1][1]};
            #pragma unroll
            for (int r = 0; r < RB; ++r)
                st.o[r][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, st.pb[r][kk]), st.o[r][dt], 0, 0, 0);
        }
        if constexpr (PREV && s < EA) {
            // pairs of the previous tile's half 1 (P^T k-steps 2, 3), before part B reads them
            #pragma unroll
            for (int u = 0; u < PPA; ++u)
                #pragma unroll
                for (int r = 0; r < RB; ++r) {
                    const int i = s * PPA + u;
                    st.pb[r][2 + (i >> 2)][i & 3] = exp_pair(s1p[r][2 * i], s1p[r][2 * i + 1], c, st.msc[r], psa[r]);
                }
        }
        if constexpr (PREV && s == EA - 1) {
            #pragma unroll
            for (int r = 0; r < RB; ++r) st.l_run[r] += psa[r];
        }
        if constexpr (CUR && s >= SA - NC && s < SA) conv(s - (SA - NC));
        if constexpr (CUR && s == SA + 1) {
            #pragma unroll
            for (int r = 0; r < RB; ++r)
                if (mk[r].masked) {
                    #pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int k0 = key_of(0, e), k1 = key_of(1, e) - 32;
                        st.s0[r][e] = ((mk[r].vis_lo >> k0) & 1u) ? st.s0[r][e] : kNegInf;
                        s1[r][e] = ((mk[r].vis_hi >> k1) & 1u) ? s1[r][e] : kNegInf;
                    }
                }
        }
        if constexpr (CUR && s >= SA + 1 && s < SA + 5) {
            constexpr int q = s - SA - 1, r0 = (q & 1) * 8;
            #pragma unroll
            for (int r = 0; r < RB; ++r) {
                const f32x16 &v = score(std::integral_constant<int, (q >> 1)>{}, r);
                const float a = max3(v[r0], v[r0 + 1], v[r0 + 2]);
                const float b = max3(v[r0 + 3], v[r0 + 4], v[r0 + 5]);
                m8[r][q] = max3(a, b, max3(v[r0 + 6], v[r0 + 7], v[r0 + 7]));
                tie(m8[r][q]);
            }
        }
        if constexpr (CUR && s == SA + 5) {
            // the running max is raised only when a score exceeds it by more than
            // kRescaleSlack (log2 units); O is rescaled after this period's products
            #pragma unroll
            for (int r = 0; r < RB; ++r) {
                const float tmax = halves_max(max3(m8[r][0], m8[r][1], max3(m8[r][2], m8[r][3], m8[r][3])));
                const bool raise = tmax * c > st.m_run[r] * c + kRescaleSlack;
                any_raise[r] = __any(raise);
                if (any_raise[r]) {
                    const float m_new = raise ? tmax : st.m_run[r];
                    alpha[r] = (st.m_run[r] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f((st.m_run[r] - m_new) * c);
                    st.l_run[r] *= alpha[r];
                    st.m_run[r] = m_new;
                }
                st.msc[r] = (st.m_run[r] == kNegInf) ? 0.f : st.m_run[r] * c;
            }
        }
        if constexpr (CUR && s >= SA + B0) {
            // pairs of half 0: k-step 0 from slot NDT of part B on, 1 from slot 2 NDT on, whose
            // products before that read the previous tile's
            constexpr int n = SB - B0, q = s - SA - B0;
            #pragma unroll
            for (int i = 8 * q / n; i < 8 * (q + 1) / n; ++i)
                #pragma unroll
                for (int r = 0; r < RB; ++r)
                    st.pb[r][i >> 2][i & 3] = exp_pair(st.s0[r][2 * i], st.s0[r][2 * i + 1], c, st.msc[r], psb[r]);
        }
        if constexpr (CUR && s >= NSLOT - NC) conv(NC + s - (NSLOT - NC));
        __builtin_amdgcn_sched_barrier(0);
    }, std::make_integer_sequence<int, NSLOT>{});
    if (CUR) {
        #pragma unroll
        for (int r = 0; r < RB; ++r) {
            st.l_run[r] += psb[r];
            if (any_raise[r]) {
                #pragma unroll
                for (int dt = 0; dt < NDT; ++dt)
                    #pragma unroll
                    for (int e = 0; e < 16; ++e) st.o[r][dt][e] *= alpha[r];
            }
        }
    }
}

template <int D, int RB>
__global__ __launch_bounds__(4 * kWave) void kv4_wide_kernel(Kv4AttnParams p) {
    using Gm = Geo<D>;
    constexpr int NW = 4, NT = NW * kWave;
    constexpr int NKS = D / 16, NDT = D / 32, C = Gm::kChunks, NC = D / 32;
    constexpr int kBlocks = Gm::kBlocksPerTile / NW;       // 1 KB blocks of a tree tile per wave, K or V
    constexpr int KPB = Gm::kKeysPerBlock;

    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    const int wave_u = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5, col = lane & 31;
    const int g4 = lane >> 4, c16 = lane & 15;
    const int w = xcd_contiguous_id(blockIdx.x, p.num_wg);

    build_cumulative<NT>(p);

    const Shares sh(g_cum[p.B], p.num_wg);
    const int start = sh.start_of(w), end = sh.start_of(w + 1);
    const unsigned ring = lds_addr(g_ring);
    // lane-constant parts of the LDS fragment addresses (see swz)
    const unsigned k_lane = col * Gm::kRowBytes + ((half ^ swz<C>(col % C)) << 4);
    const int va = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const int vb = half * 4 + ((lane & 15) >> 2);
    const unsigned v_lane = vb * Gm::kRowBytes + ((va ^ swz<C>(vb)) << 4) + (lane & 1) * 8;

    int pos = start;
    int anc_b = -1;
    if (start >= end && tid == 0) p.ws_desc[w * 4] = -1;
    while (pos < end) {
        Piece pc;
        if (!next_piece(p, sh, w, start, end, pos, pc)) continue;
        const int b = pc.b, g = pc.g, ntp = pc.ntp, t0 = pc.t0, t_end = pc.t_end;
        const bool paths = needs_paths(p, pc) && anc_b != b;
        int par = -1;
        if (paths && wave_u == 0 && p.N <= kWave && lane < p.N) par = p.parent[(size_t)b * p.N + lane];

        // ---- codes: key 16 wave + c16 of a tile, D/4 values from (D/4) g4 on
        const int kkey = 16 * wave_u + c16;
        auto pos_of = [&](int t) { return pc.real(t) * KT + kkey; };
        const int32_t *pages = p.page_table + (size_t)b * p.max_pages;
        auto id_of = [&](int t) { return pages[min(max(pos_of(t), 0) >> p.p_shift, p.max_pages - 1)]; };
        auto row_at = [&](int t, int id) { return t < min(t_end, ntp) ? row_of(p, g, pos_of(t), id, pc.L, pc.sp) : -1ll; };
        Part4<D> rk[2], rv[2];             // K of tile t in rk[t & 1], V in rv[t & 1]
        long long row[2];                  // the rows of the tiles whose V is still to be loaded
        int id[2];
        #pragma unroll
        for (int i = 0; i < 2; ++i) id[i] = id_of(t0 + i);

        // ---- this wave's query rows: a row past the unit's last one loads the unit's first
        WideState<D, RB> st;
        int node[RB], hq[RB];
        bool row_ok[RB];
        #pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int first = pc.rb * p.rows_per_block, at = first + (wave_u * RB + r) * 32 + col;
            row_ok[r] = at < pc.rows_b;
            const int qrow = row_ok[r] ? at : first;
            node[r] = qrow / p.G;
            hq[r] = g * p.G + qrow % p.G;
            const uint16_t *qp = p.q + (((size_t)b * p.N + node[r]) * p.Hq + hq[r]) * D + half * 8;
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                st.qf[r][ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8 *>(qp + ks * 16));
            #pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
                #pragma unroll
                for (int e = 0; e < 16; ++e) st.o[r][dt][e] = 0.f;
            st.m_run[r] = kNegInf;
            st.msc[r] = 0.f;
            st.l_run[r] = 0.f;
        }

        // ---- LDS places: converted tile t in stage t & 1 (K, then V); tree tile u in stage
        // 2 + u, the third and fourth in stages ntp & 1 and (ntp + 1) & 1 (their turn)
        auto stage_of = [&](int t) { return t < ntp ? t & 1 : t - ntp < 2 ? 2 + t - ntp : t & 1; };
        auto load_tree = [&](int t) {
            unsigned char *dst = g_ring + stage_of(t) * Gm::kStageBytes;
            #pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const int blk = wave_u * kBlocks + i, key = blk * KPB + lane / C, j = (t - ntp) * KT + key;
                // a slot past the sequence's nodes reads node 0's row (finite, masked)
                const size_t at = (((size_t)b * p.N + (j < pc.nodes ? j : 0)) * p.Hkv + g) * D +
                                  ((lane % C) ^ swz<C>(key % C)) * 8;
                __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)(p.k_tree + at), (LDS_AS void *)(dst + blk * 1024),
                                                 16, 0, 0);
                __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)(p.v_tree + at),
                                                 (LDS_AS void *)(dst + Gm::kTileBytes + blk * 1024), 16, 0, 0);
            }
        };
        auto krow = [&](int t) { return g_ring + (t & 1) * Gm::kStageBytes + kkey * Gm::kRowBytes; };
        auto vrow = [&](int t) { return krow(t) + Gm::kTileBytes; };

        // first loads: K of the first three tiles, V of the first two; the first tile's K is
        // converted before the loop
        row[0] = row_at(t0, id[0]);
        row[1] = row_at(t0 + 1, id[1]);
        id[0] = id_of(t0 + 2);
        id[1] = id_of(t0 + 3);
        Part4<D> k0;
        load_part<D>(k0, p, row[0], false, g4);
        load_part<D>(rk[1], p, row[1], false, g4);
        load_part<D>(rv[0], p, row[0], true, g4);
        load_part<D>(rv[1], p, row[1], true, g4);
        row[0] = row_at(t0 + 2, id[0]);
        load_part<D>(rk[0], p, row[0], false, g4);
        id[0] = id_of(t0 + 4);
        if (t_end > ntp)
            for (int t = max(ntp, t0); t < t_end; ++t)
                if (t0 >= ntp || t < ntp + 2) load_tree(t);
        if (paths) {
            if (wave_u == 0) {
                tie(par);
                if (p.N <= kWave) build_ancestor_masks_wave(p, par);
                else build_ancestor_masks_wave_lds(p, b);
            }
            anc_b = b;
        }
        if (t0 < ntp) {
            #pragma unroll
            for (int i = 0; i < NC; ++i) convert_chunk<D>(k0, krow(t0), g4 * NC, kkey, i);
        }

        f32x16 s1[2][RB];
        TileMask mk[RB];
        // Opens the period of tile t: the converted parts of every wave are in place, and the
        // tree tiles that it or the one before reads; then the tile's mask.
        auto open = [&](int t) {
            if (t >= ntp) wait_vmcnt<0>();
            lds_barrier();
            if (t >= t_end) return;
            if (t0 < ntp && t >= ntp && t < ntp + 2 && t + 2 < t_end) load_tree(t + 2);
            const int base = pc.real(t) * KT;
            const bool tree = t >= ntp;
            const bool masked = tree || base + KT > pc.L || !window_clear(pc.sp, base, p.N);
            #pragma unroll
            for (int r = 0; r < RB; ++r) {
                mk[r].masked = masked;
                if (masked) {
                    const unsigned long long vis = (tree ? window_path(g_anc[node[r]], t - ntp, pc.L, p)
                                                         : prefix_bits(p, pc, base, node[r])) >> (half * 4);
                    mk[r].vis_lo = (unsigned)vis;
                    mk[r].vis_hi = (unsigned)(vis >> 32);
                }
            }
        };
        auto kaddr = [&](int t) { return ring + stage_of(t) * Gm::kStageBytes + k_lane; };
        auto vaddr = [&](int t) { return ring + stage_of(t) * Gm::kStageBytes + Gm::kTileBytes + v_lane; };
        // Period of tile t = t0 + j, j of parity PAR: converts K_{t+1} (rk[1 - PAR]) and V_t
        // (rv[PAR]) and loads K_{t+3} and V_{t+2} in their place.
        auto period = [&](auto par_, auto prev_, int t) {
            constexpr int PAR = decltype(par_)::value;
            open(t);
            wide_period<D, RB, decltype(prev_)::value, true>(
                st, s1[1 - PAR], s1[PAR], kaddr(t), decltype(prev_)::value ? vaddr(t - 1) : 0u, mk, p.scale_log2,
                [&](int i) {
                    if (i < NC) {
                        if (t + 1 < min(t_end, ntp)) convert_chunk<D>(rk[1 - PAR], krow(t + 1), g4 * NC, kkey, i);
                    } else if (t < ntp) {
                        convert_chunk<D>(rv[PAR], vrow(t), g4 * NC, kkey, i - NC);
                    }
                });
            // V_{t+2} from the row found for K_{t+2}, then K_{t+3}
            load_part<D>(rv[PAR], p, row[PAR], true, g4);
            row[1 - PAR] = row_at(t + 3, id[1 - PAR]);
            load_part<D>(rk[1 - PAR], p, row[1 - PAR], false, g4);
            id[1 - PAR] = id_of(t + 5);
        };
        using E_ = std::integral_constant<int, 0>;
        using O_ = std::integral_constant<int, 1>;
        period(E_{}, std::false_type{}, t0);
        int t = t0 + 1;
        for (; t + 1 < t_end; t += 2) {
            period(O_{}, std::true_type{}, t);
            period(E_{}, std::true_type{}, t + 1);
        }
        const bool odd = t < t_end;
        if (odd) period(O_{}, std::true_type{}, t);
        // PV of the last tile
        open(t_end);
        if (odd)
            wide_period<D, RB, true, false>(st, s1[1], s1[0], 0u, vaddr(t_end - 1), mk, p.scale_log2, [](int) {});
        else
            wide_period<D, RB, true, false>(st, s1[0], s1[1], 0u, vaddr(t_end - 1), mk, p.scale_log2, [](int) {});
        __syncthreads();

        // ---- the normalised rows leave through this wave's part of the idle ring, transposed
        // there so that every store writes whole rows; a piece of a split unit as fp16 times a
        // power of two per row
        constexpr int kPitch = D * 2 + 16, kRowChunks = D / 8, kRowsPerPass = kWave / kRowChunks;
        unsigned char *wbuf = g_ring + wave_u * 32 * kPitch;
        #pragma unroll
        for (int r = 0; r < RB; ++r) {
            const float l_tot = halves_sum(st.l_run[r]);
            const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
            float unscale = 1.f, scaled = inv;
            if (!pc.complete) {
                const float top = row_top(
                    [&](auto take) {
                        #pragma unroll
                        for (int dt = 0; dt < NDT; ++dt)
                            #pragma unroll
                            for (int e = 0; e < 16; ++e) take(st.o[r][dt][e]);
                    },
                    halves_max);
                scaled *= part_scale(top * inv, unscale);
            }
            #pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
                #pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    bf16x4 v;
                    f16x4 f;
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[i] = (__bf16)(st.o[r][dt][q4 * 4 + i] * inv);
                        f[i] = (_Float16)(st.o[r][dt][q4 * 4 + i] * scaled);
                    }
                    if (!pc.complete) v = __builtin_bit_cast(bf16x4, f);
                    *reinterpret_cast<bf16x4 *>(wbuf + col * kPitch + (dt * 32 + q4 * 8 + half * 4) * 2) = v;
                }
            #pragma unroll
            for (int k = 0; k < 32 / kRowsPerPass; ++k) {
                const int rr = k * kRowsPerPass + lane / kRowChunks, ch = lane % kRowChunks;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(wbuf + rr * kPitch + ch * 16);
                const int rl = (wave_u * RB + r) * 32 + rr;          // row within the unit's block
                if (pc.complete) {
                    const int ur = pc.rb * p.rows_per_block + rl;
                    if (ur < pc.rows_b) {
                        const int nd = ur / p.G, h = g * p.G + ur % p.G;
                        *reinterpret_cast<u32x4 *>(p.out + (((size_t)b * p.N + nd) * p.Hq + h) * D + ch * 8) = v;
                    }
                } else {
                    *reinterpret_cast<u32x4 *>(p.ws_o + ((size_t)pc.slot * p.rows_per_block + rl) * D + ch * 8) = v;
                }
            }
            if (half == 0) {
                if (pc.complete) {
                    if (row_ok[r] && p.lse)
                        p.lse[((size_t)b * p.N + node[r]) * p.Hq + hq[r]] =
                            st.m_run[r] * p.scale + __builtin_amdgcn_logf(l_tot) * kLn2;
                } else {
                    const int rl = (wave_u * RB + r) * 32 + col;
                    *reinterpret_cast<f32x4 *>(p.ws_ml + ((size_t)pc.slot * p.rows_per_block + rl) * 4) =
                        f32x4{st.m_run[r] == kNegInf ? kNegInf : st.m_run[r] * p.scale_log2, l_tot, unscale, 0.f};
                }
            }
        }
        __syncthreads();                   // the ring is refilled by the next piece
    }

    clear_padding<D, NT>(p, w);
}

template <int D>
hipError_t launch_d(const Kv4AttnParams &p, hipStream_t s) {
    auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(p.num_wg), dim3(4 * kWave), s, p); };
    if (p.rows_per_block == 128) return go(kv4_wide_kernel<D, 1>);
    if (p.rows_per_block == 256) return go(kv4_wide_kernel<D, 2>);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv4_wide(const Kv4AttnParams &p, int head_dim, hipStream_t s) {
    if (head_dim == 64) return launch_d<64>(p, s);
    if (head_dim == 128) return launch_d<128>(p, s);
    return hipErrorInvalidValue;
}

}  // namespace tv
