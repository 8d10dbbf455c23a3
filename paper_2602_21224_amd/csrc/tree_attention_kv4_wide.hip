// Tree-masked attention over a prefix held in 4 bits for units of many query rows, for
// gfx950 (tree_attention_kv4.hip has those of few).
//
// Such a call is bound by the matrix cores and the softmax between their instructions, not
// by bytes. A unit's row block is 256 rows (eight waves of 32; up to 128 rows: four), which
// step through the block's 64-key tiles together, and each tile is converted once per
// workgroup into a bf16 tile in LDS: from there on it is the bf16 attention's period
// (tile_period: S_t^T = K_t Q^T and O^T += V_{t-1}^T P_{t-1}^T with the softmax between their
// MFMAs). K_{t+1} goes where K_{t-1} was and V_t where V_{t-2} was, both read before the
// barrier that opens period t, so two tiles of each are enough.
//
// A wave converts the keys 64/NW w .. of K_{t+1} and V_t at the end of its period t, a lane
// a block of 32 values: 16 bytes of codes and a scale byte. It has loaded them itself, direct
// to LDS three periods ahead, the same number of loads every time, so its own wait, for a
// constant count, is enough. (Loads into registers, which the compiler waits for, made every
// second period wait for all of them.) Its keys of a tile lie in one page, whose id is a
// scalar load; with smaller pages (SMALL) every lane has its own, by a direct-to-LDS load
// two periods before the codes.
// The tree's rows are bf16 already and come straight into the converted tiles' places, a
// period ahead.
//
// Measured (16 x 64 nodes, 4 heads per KV head, over 1024-4096 tokens): 64-70 us, 10 of them
// for joining the split rows. A tile costs a CU about 5000 cycles, of which the matrix cores
// take 2048, the softmax, masks and conversions 3000 and LDS 2450; 22000 of 133000 cycles are
// outside the tiles. Waves in their products go before those that convert (s_setprio): 4 x 64
// nodes over 32768 tokens 167 -> 160 us, 4 x 256 nodes 600 -> 573 (over bf16: 568). Four waves of
// 64 rows each, which halve the operand reads from LDS, took 88 us where this took 66: one wave
// per SIMD issues an instruction every 6.8 cycles, and its vector work was as long as the period.
// Blocks of 64 rows whose waves each convert tiles of their own: 299.
#include "tree_attention_kv4.h"

namespace tv {
namespace {

__device__ __forceinline__ unsigned read_dword(unsigned addr) {
    unsigned x;
    asm volatile("ds_read_b32 %0, %1" : "=v"(x) : "v"(addr));
    return x;
}
__device__ __forceinline__ u32x4 read_codes(unsigned addr) {
    u32x4 x;
    asm volatile("ds_read_b128 %0, %1" : "=v"(x) : "v"(addr));
    return x;
}
// A store beside loads in flight to other places of the same array, for which the compiler
// would wait.
__device__ __forceinline__ void write_chunk(unsigned addr, const bf16x8 &x) {
    asm volatile("ds_write_b128 %0, %1" ::"v"(addr), "v"(__builtin_bit_cast(u32x4, x)));
}

// The blocks of 32 values that a wave converts per period, one per lane and step: half of
// them of K, then those of V.
template <int D, int NW>
struct Share4 {
    static constexpr int kBlocks = D / kBlock4;                    // per row
    static constexpr int kTasks = 2 * (KT / NW) * kBlocks;
    static constexpr int kSteps = kTasks > kWave ? kTasks / kWave : 1;
    static constexpr int kBytes = kSteps * (kWave * 16 + kWave * 4);   // codes, and a dword of scales each
    static constexpr int kLoads = 2 * kSteps;
    static constexpr int kDepth = 4;
    static constexpr int kIdDepth = 4;
    bool is_v;
    int key, blk;                          // key within the wave's
    __device__ __forceinline__ Share4(int lane, int step) {
        const int task = (step * kWave + lane) % kTasks;           // lanes past the last task repeat
        is_v = task >= kTasks / 2;
        const int i = task % (kTasks / 2);
        key = i / kBlocks;
        blk = i % kBlocks;
    }
};

template <int D, int NW, bool SMALL>
__global__ __launch_bounds__(NW * kWave) void kv4_wide_kernel(Kv4AttnParams p) {
    using Gm = Geo<D>;
    using Sh = Share4<D, NW>;
    constexpr int NT = NW * kWave;
    constexpr int NKS = D / 16, NDT = D / 32, C = Gm::kChunks;
    constexpr int kTreeLoads = Gm::kBlocksPerTile / NW;    // 1 KB blocks of a tree tile per wave, K or V
    constexpr int KPB = Gm::kKeysPerBlock;
    constexpr int KPW = KT / NW;                           // keys of a tile that a wave converts
    constexpr int L4 = Sh::kLoads, LID = SMALL ? Sh::kSteps : 0;   // its loads per period: codes, ids
    constexpr int kRaw = NW * Sh::kDepth * Sh::kBytes;
    static_assert(2 * Gm::kStageBytes + kRaw + NW * Sh::kIdDepth * Sh::kSteps * 256 <= (int)sizeof(g_ring),
                  "two tiles of K and V, raw blocks and page ids fit");

    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    const int wave_u = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int half = lane >> 5, col = lane & 31;
    const int w = xcd_contiguous_id(blockIdx.x, p.num_wg);

    build_cumulative(p, [&](int L, int nodes) { return sequence_tiles(p, L, nodes); });

    const Shares sh(g_cum[p.B], p.num_wg);
    const int start = sh.start_of(w), end = sh.start_of(w + 1);
    const unsigned ring = lds_addr(g_ring);
    unsigned char *raw = g_ring + 2 * Gm::kStageBytes + wave_u * Sh::kDepth * Sh::kBytes;
    unsigned char *id_ring = g_ring + 2 * Gm::kStageBytes + kRaw + wave_u * Sh::kIdDepth * Sh::kSteps * 256;
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

        // ---- loads of this wave's share of period u: K of tile u + 1, V of tile u (past the
        // prefix or the piece, or without a page: the cache's first row)
        const int32_t *pages = p.page_table + (size_t)b * p.max_pages;
        const int tp_end = min(t_end, ntp);
        auto page_at = [&](int at) { return min(max(at, 0) >> p.p_shift, p.max_pages - 1); };
        auto load_ids = [&](int u) {
            #pragma unroll
            for (int i = 0; i < Sh::kSteps; ++i) {
                const Sh mine(lane, i);
                const int at = pc.real(u + !mine.is_v) * KT + wave_u * KPW + mine.key;
                __builtin_amdgcn_global_load_lds(
                    (const GLOBAL_AS void *)(pages + page_at(at)),
                    (LDS_AS void *)(id_ring + ((u & (Sh::kIdDepth - 1)) * Sh::kSteps + i) * 256), 4, 0, 0);
            }
        };
        auto id_of = [&](int t) { return ((const CONST_AS int32_t *)pages)[page_at(pc.real(t) * KT + wave_u * KPW)]; };
        // first row of the wave's keys of tile t on page id
        auto first_row = [&](int t, int id) {
            const int at = pc.real(t) * KT + wave_u * KPW;
            const long long row = (((long long)(unsigned)id * (unsigned)p.Hkv + (unsigned)g) << p.p_shift) + (at & (p.P - 1));
            return t >= t0 && t < tp_end && (unsigned)id < (unsigned)p.num_pages ? row : 0ll;
        };
        auto load_from = [&](int u, int i, const uint8_t *codes, const uint8_t *scales) {
            unsigned char *to = raw + (u & (Sh::kDepth - 1)) * Sh::kBytes + i * 1280;
            __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)codes, (LDS_AS void *)to, 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)scales, (LDS_AS void *)(to + 1024), 4, 0, 0);
        };
        long long row_v = 0;               // of the tile whose K was loaded last
        int id_k = 0;                      // page id of the next one
        auto load_codes = [&](int u) {
            if constexpr (!SMALL) {
                const long long row_k = first_row(u + 1, id_k);
                #pragma unroll
                for (int i = 0; i < Sh::kSteps; ++i) {
                    const Sh mine(lane, i);
                    const uint8_t *codes = mine.is_v ? p.v4 + row_v * (D / 2) : p.k4 + row_k * (D / 2);
                    const uint8_t *scales = p.scales + (mine.is_v ? row_v : row_k) * (D / 16);
                    load_from(u, i, codes + (mine.key * (D / 2) + mine.blk * 16),
                              scales + (mine.key * (D / 16) + (D == 128 && mine.is_v ? 4 : 0)));
                }
                row_v = row_k;
                id_k = id_of(u + 2);
            } else {
                #pragma unroll
                for (int i = 0; i < Sh::kSteps; ++i) {
                    const Sh mine(lane, i);
                    unsigned id = read_dword(lds_addr(id_ring) + ((u & (Sh::kIdDepth - 1)) * Sh::kSteps + i) * 256 + lane * 4);
                    lds_wait<0>();
                    tie(id);
                    const int t = u + !mine.is_v, at = pc.real(t) * KT + wave_u * KPW + mine.key;
                    const long long row =
                        max(t >= t0 && t < tp_end ? row_of(p, g, at, (int)id, pc.L, pc.sp) : -1ll, 0ll);
                    load_from(u, i, (mine.is_v ? p.v4 : p.k4) + row * (D / 2) + mine.blk * 16,
                              p.scales + row * (D / 16) + (D == 128 && mine.is_v ? 4 : 0));
                }
            }
        };
        if constexpr (SMALL) {
            #pragma unroll
            for (int i = -1; i < 3; ++i) load_ids(t0 + i);
        } else {
            id_k = id_of(t0);
        }

        // ---- this wave's 32 query rows: a row past the unit's last one loads the unit's first
        const int row0 = pc.rb * p.rows_per_block, row_at = row0 + wave_u * kRowsPerWave + col;
        const int qrow = row_at < pc.rows_b ? row_at : row0;
        const int node = node_of(p, qrow), hq = g * p.G + qrow - node * p.G;
        WaveState<D> st;
        {
            const uint16_t *qp = p.q + (((size_t)b * p.N + node) * p.Hq + hq) * D + half * 8;
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                st.qf[ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8 *>(qp + ks * 16));
            #pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
                #pragma unroll
                for (int e = 0; e < 16; ++e) st.o[dt][e] = 0.f;
            st.m_run = kNegInf;
            st.msc = 0.f;
            st.l_run = 0.f;
        }

        // ---- tile t, converted or of the tree, is in stage t & 1 (K, then V)
        auto load_tree = [&](int t, bool is_v) {
            int ln = lane;
            tie(ln);                       // addresses are made here, not kept from the piece's start
            unsigned char *dst = g_ring + (t & 1) * Gm::kStageBytes + (is_v ? Gm::kTileBytes : 0);
            #pragma unroll
            for (int i = 0; i < kTreeLoads; ++i) {
                const int block = wave_u * kTreeLoads + i, key = block * KPB + ln / C, j = (t - ntp) * KT + key;
                // a slot past the sequence's nodes reads node 0's row (finite, masked)
                const size_t at = (((size_t)b * p.N + (j < pc.nodes ? j : 0)) * p.Hkv + g) * D +
                                  ((ln % C) ^ swz<C>(key % C)) * 8;
                __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)((is_v ? p.v_tree : p.k_tree) + at),
                                                 (LDS_AS void *)(dst + block * 1024), 16, 0, 0);
            }
        };
        // Conversion of the share of period u. A key that no node sees counts as zeros.
        auto convert = [&](int u) {
            const int base_k = pc.real(u + 1) * KT, base_v = pc.real(u) * KT;
            auto clear = [&](int base) { return base + KT <= pc.L && (base >= pc.sp.lo || base + KT <= pc.sp.sinks); };
            const bool all = clear(base_k) && clear(base_v);
            #pragma unroll
            for (int i = 0; i < Sh::kSteps; ++i) {
                const Sh mine(lane, i);
                const unsigned from = lds_addr(raw) + (u & (Sh::kDepth - 1)) * Sh::kBytes + i * 1280;
                u32x4 x = read_codes(from + lane * 16);
                unsigned sc = read_dword(from + 1024 + lane * 4);
                const int key = wave_u * KPW + mine.key;
                // stages (u + 1) & 1 for K and u & 1 for V
                const unsigned to = ring + ((key * Gm::kRowBytes + (((mine.blk * 4) ^ swz<C>(key % C)) << 4) +
                                             (mine.is_v ? Gm::kTileBytes : Gm::kStageBytes)) ^
                                            ((u & 1) * Gm::kStageBytes));
                lds_wait<0>();
                tie(x);
                tie(sc);
                unsigned e = (sc >> (8 * (mine.blk + (D == 64 && mine.is_v ? 2 : 0)))) & 255u;
                if (!all) {
                    const int at = (mine.is_v ? base_v : base_k) + key;
                    if (!(at < pc.L && (at >= pc.sp.lo || at < pc.sp.sinks))) {
                        x = u32x4{0, 0, 0, 0};
                        e = 127;
                    }
                }
                if (u + !mine.is_v < ntp) {
                    #pragma unroll
                    for (int q = 0; q < 4; ++q) write_chunk(to ^ (q << 4), from4x8(x[q], scale4(e)));
                }
            }
        };

        if (paths && wave_u == 0) {
            tie(par);
            if (p.N <= kWave) build_ancestor_masks_wave(p, par);
            else build_ancestor_masks_wave_lds(p, b);
        }
        if (paths) anc_b = b;
        // in the order of the loop below, whose waits count: codes of period u, ids of u + 2
        if (SMALL) wait_vmcnt<0>();
        load_codes(t0 - 1);
        load_codes(t0);
        if (SMALL) load_ids(t0 + 3);
        load_codes(t0 + 1);
        if (SMALL) load_ids(t0 + 4);
        load_codes(t0 + 2);
        if (t0 < ntp) {
            wait_vmcnt<3 * L4 + 2 * LID>();
            convert(t0 - 1);
        } else {
            load_tree(t0, false);
        }

        f32x16 s0, s1;
        TileMask mk;
        // Opens the period of tile t: K_t and V_{t-1} of every wave are in place; then the loads
        // of tree rows that go where K_{t-1} and V_{t-2} were, and the tile's mask.
        auto open = [&](int t) {
            if (t >= ntp) wait_vmcnt<0>();
            lds_barrier();
            if (t >= t_end) return;
            if (t + 1 >= ntp && t + 1 < t_end) load_tree(t + 1, false);
            if (t >= ntp) load_tree(t, true);
            const int base = pc.real(t) * KT;
            const bool tree = t >= ntp;
            mk.masked = tree || base + KT > pc.L || !window_clear(pc.sp, base, p.N);
            if (mk.masked) {
                const unsigned long long vis =
                    (tree ? window_path(g_anc[node], t - ntp, pc.L, p) : prefix_bits(p, pc, base, node)) >> (half * 4);
                mk.vis_lo = (unsigned)vis;
                mk.vis_hi = (unsigned)(vis >> 32);
            }
        };
        auto kaddr = [&](int t) { return ring + (t & 1) * Gm::kStageBytes + k_lane; };
        auto vaddr = [&](int t) { return ring + (t & 1) * Gm::kStageBytes + Gm::kTileBytes + v_lane; };
        auto close = [&](int t) {
            // the codes of period t: behind them those of two periods, and ids
            if (t < ntp) {
                wait_vmcnt<2 * (L4 + LID)>();
                convert(t);
            }
            if constexpr (SMALL) {
                // the ids of period t + 3: behind them one period's ids and two periods' codes
                wait_vmcnt<2 * L4 + LID>();
                load_ids(t + 5);
            }
            load_codes(t + 3);
        };
        open(t0);
        tile_period<D, false, true>(st, s0, s1, kaddr(t0), 0u, mk, p.scale_log2);
        close(t0);
        for (int t = t0 + 1; t < t_end; ++t) {
            open(t);
            __builtin_amdgcn_s_setprio(1);         // products before the other waves' conversions
            tile_period<D, true, true>(st, s0, s1, kaddr(t), vaddr(t - 1), mk, p.scale_log2);
            __builtin_amdgcn_s_setprio(0);
            close(t);
        }
        open(t_end);
        tile_period<D, true, false>(st, s0, s1, 0u, vaddr(t_end - 1), mk, p.scale_log2);
        wait_vmcnt<0>();                   // no load of codes lands in what follows
        __syncthreads();

        // ---- the normalised rows leave through this wave's part of the idle ring, transposed
        // there so that every store writes whole rows; a piece of a split unit as fp16 times a
        // power of two per row
        constexpr int kPitch = D * 2 + 16, kRowChunks = D / 8, kRowsPerPass = kWave / kRowChunks;
        unsigned char *wbuf = g_ring + wave_u * 32 * kPitch;
        int ln = lane;
        tie(ln);                           // addresses are made here, not kept from the piece's start
        {
            const float l_tot = halves_sum(st.l_run);
            const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
            unsigned char *to = wbuf + (ln & 31) * kPitch + (ln >> 5) * 8;
            float unscale = 1.f;
            if (pc.complete) {
                #pragma unroll
                for (int q = 0; q < 4 * NDT; ++q) {
                    bf16x4 v;
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = (__bf16)(st.o[q >> 2][(q & 3) * 4 + i] * inv);
                    *reinterpret_cast<bf16x4 *>(to + q * 16) = v;
                }
            } else {
                const float top = row_top(
                    [&](auto take) {
                        #pragma unroll
                        for (int dt = 0; dt < NDT; ++dt)
                            #pragma unroll
                            for (int e = 0; e < 16; ++e) take(st.o[dt][e]);
                    },
                    halves_max);
                const float scaled = inv * part_scale(top * inv, unscale);
                #pragma unroll
                for (int q = 0; q < 4 * NDT; ++q) {
                    f16x4 f;
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) f[i] = (_Float16)(st.o[q >> 2][(q & 3) * 4 + i] * scaled);
                    *reinterpret_cast<f16x4 *>(to + q * 16) = f;
                }
            }
            const int rl0 = wave_u * kRowsPerWave + ln / kRowChunks, ch = ln % kRowChunks;   // within the block
            #pragma unroll
            for (int k = 0; k < 32 / kRowsPerPass; ++k) {
                const int rl = rl0 + k * kRowsPerPass;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(wbuf + (k * kRowsPerPass + ln / kRowChunks) * kPitch + ch * 16);
                if (pc.complete) {
                    const int ur = pc.rb * p.rows_per_block + rl;
                    if (ur < pc.rows_b) {
                        const int nd = node_of(p, ur), h = g * p.G + ur - nd * p.G;
                        *reinterpret_cast<u32x4 *>(p.out + (((size_t)b * p.N + nd) * p.Hq + h) * D + ch * 8) = v;
                    }
                } else {
                    *reinterpret_cast<u32x4 *>(p.ws_o + ((size_t)pc.slot * p.rows_per_block + rl) * D + ch * 8) = v;
                }
            }
            if (ln < 32) {
                const int rl = wave_u * kRowsPerWave + ln;
                if (!pc.complete)
                    *reinterpret_cast<f32x4 *>(p.ws_ml + ((size_t)pc.slot * p.rows_per_block + rl) * 4) =
                        f32x4{part_max(st.m_run, l_tot, p.scale_log2), l_tot, unscale, 0.f};
                else if (p.lse && pc.rb * p.rows_per_block + rl < pc.rows_b)
                    p.lse[((size_t)b * p.N + node) * p.Hq + hq] =
                        st.m_run * p.scale + __builtin_amdgcn_logf(l_tot) * kLn2;
            }
        }
        __syncthreads();                   // the ring is refilled by the next piece
    }

    clear_padding<D, NT>(p, w);
}

template <int D>
hipError_t launch_d(const Kv4AttnParams &p, hipStream_t s) {
    auto go = [&](auto kernel, int waves) { return launch_kernel(kernel, dim3(p.num_wg), dim3(waves * kWave), s, p); };
    if (p.rows_per_block == 128)
        return p.P < KT / 4 ? go(kv4_wide_kernel<D, 4, true>, 4) : go(kv4_wide_kernel<D, 4, false>, 4);
    if (p.rows_per_block == 256)
        return p.P < KT / 8 ? go(kv4_wide_kernel<D, 8, true>, 8) : go(kv4_wide_kernel<D, 8, false>, 8);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv4_wide(const Kv4AttnParams &p, int head_dim, hipStream_t s) {
    if (head_dim == 64) return launch_d<64>(p, s);
    if (head_dim == 128) return launch_d<128>(p, s);
    return hipErrorInvalidValue;
}

}  // namespace tv
