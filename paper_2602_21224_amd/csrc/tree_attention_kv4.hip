// Tree-masked attention over a paged prefix held in 4 bits (kv4.h), with an optional
// sliding window, for gfx950.
//
// The function is tree_verify_attention's, with the values that the codes stand for in
// place of the cache's rows. A key of a KV head is D/2 bytes of codes and D/32 scale bytes
// for K and the same for V, 136 bytes at head size 128 where bf16 takes 512.
//
// Work decomposition: units (sequence, KV head, block of 16 NR query rows), their 64-key
// tiles laid end to end and shared out equally over the workgroups as in
// tree_attention.hip. Within a piece the workgroup's four waves take its tiles in turn, each by
// itself: no barrier until the piece ends, where the waves' (max, sum, O) meet in LDS. Two
// workgroups per CU, so that one streams while the other finds and starts a piece.
//
// One tile of one wave, v_mfma_f32_16x16x32_bf16 throughout. Lane l = 16 g + c:
//   S^T = K Q^T: the lane holds key 16 kb + c of every key block kb, and of it the D/4
//     values from (D/4) g on, which are one load of 16 (8) bytes of codes. That order of
//     the head dimension is not the operand's own, but the sum over it is the same in any
//     order, so Q's fragments are loaded in the same one and K needs no shuffle: eight
//     codes become one operand by four conversions. (v_mfma_scale_f32_16x16x128_f8f6f4, which
//     takes the codes and scales as they lie and Q as two fp8 parts, was built and is no
//     faster: the conversions are not what bounds this.)
//   O^T += V^T P^T: the operand wants eight keys of one column per lane. The lane
//     converts the same part of V's row and stores it to a row-major half tile of the wave's
//     own in LDS (16-byte chunks swizzled by the key), and ds_read_b64_tr_b16 reads it
//     transposed, with the key order that the scores' accumulators have.
// Bound by the stream of codes where prefixes are long: 64 sequences of 2048-8192 tokens, one
// node x 4 heads per KV head, 79-82 us, 363 MB read at 4.5 TB/s; 4 x 4 nodes over 98304-131072
// tokens 107 us, 4.7 TB/s (a copy reaches 4.8). 16 x 12 nodes x 32 heads over 256-2048 tokens,
// about one unit per workgroup, take 34 us where the bytes take 18, one sequence of 2048 tokens
// 14: the way to the first tile (lengths, search, page ids) 2.4 us, two tiles 3, the waves'
// meeting 1.8, the launch, the joining kernel 4.
// With four waves per CU (one workgroup, a set of registers more in flight) these were 98, 111,
// 50 and 19; loading the first codes before the root paths are found, and the tree's tiles first,
// 90 instead of 80 and 36 instead of 33.
// The registers that held a tile's codes of K take the next tile's as soon as its scores are
// under way, those of V when V is in LDS: loads are on their way for most of a tile's time, and
// with two sets of registers (a set more in flight) a wave spilled. (Of the instances, those for 32
// rows of head size 128 spill 4 registers, 11 with pages of fewer than 16 keys: in the set-up of
// trees of more than 64 nodes, not in the tiles.)
#include "tree_attention_kv4.h"

namespace tv {
namespace {

// A wave's raw loads of one prefix tile: D/4 values of K and of V of one key per block.
template <int D>
struct Raw4 {
    static constexpr int W = D / 32;                   // dwords of codes
    unsigned k[4][W], v[4][W];
    unsigned ks[4], vs[4];                             // scale bytes
};

template <int D, int NR>
struct StreamState {
    static constexpr int NKS = D / 32;                 // k-steps over the head dim (S)
    static constexpr int NDB = D / 16;                 // 16-wide head-dim blocks of O^T
    bf16x8 qf[NR][NKS];
    f32x4 o[NR][NDB];
    float m_run[NR], l_run[NR];
};

constexpr int kStreamWaves = 4;
constexpr int kStreamWgPerCu = 2;
__shared__ __attribute__((aligned(1024))) unsigned char g_half[kStreamWaves * Geo<128>::kTileBytes / 2];
__shared__ float g_ml[kStreamWaves][16][2];

// Rows of the cache (of one KV head's tokens) that hold the key blocks of the prefix tile at
// position `base`; a block without a page takes the cache's first rows. SMALL: pages of fewer
// than 16 keys, so every lane has its own.
template <bool SMALL>
__device__ __forceinline__ void find_rows(const Kv4AttnParams &p, const Piece &pc, int base, int c, long long (&row)[4]) {
    const int32_t *pages = p.page_table + (size_t)pc.b * p.max_pages;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        const int at = base + 16 * kb + (SMALL ? c : 0);
        const int page = min(at >> p.p_shift, p.max_pages - 1);
        const int id = SMALL ? pages[page] : ((const CONST_AS int32_t *)pages)[page];
        row[kb] = (((long long)(unsigned)id * (unsigned)p.Hkv + (unsigned)pc.g) << p.p_shift) + (at & (p.P - 1));
        if ((unsigned)id >= (unsigned)p.num_pages) row[kb] = 0;
    }
}

template <int D, bool SMALL>
__device__ __forceinline__ void load_part(const Kv4AttnParams &p, const long long (&row)[4], bool is_v, int lane,
                                          unsigned (&x)[4][D / 32], unsigned (&e)[4]) {
    const int c = SMALL ? 0 : lane & 15, g = lane >> 4;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        load_dwords(x[kb], (is_v ? p.v4 : p.k4) + row[kb] * (D / 2) + (unsigned)(c * (D / 2) + g * (D / 8)));
        e[kb] = (p.scales + row[kb] * (D / 16))[(unsigned)(c * (D / 16) + (is_v ? D / kBlock4 : 0) + g * (D / 4) / kBlock4)];
    }
}

// V of the keys that no node sees (past the prefix, behind the window) counts as zeros: their
// weight is 0, which does not hide a NaN. (K's scores are replaced.)
template <int D>
__device__ __forceinline__ void drop_unseen(const Piece &pc, int base, int c, Raw4<D> &r) {
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        const int at = base + 16 * kb + c;
        if (!(at < pc.L && (at >= pc.sp.lo || at < pc.sp.sinks))) {
            #pragma unroll
            for (int w = 0; w < Raw4<D>::W; ++w) r.v[kb][w] = 0;
            r.vs[kb] = 127;
        }
    }
}

// One tile: kfrag(kb, t) and vfrag(kb, t) give eight values of the lane's key of block kb,
// from head-dim index (D/4) g + 8 t on; `vis` the keys that the lane's row of tile nr sees.
// k_done and v_done are called when the lane's codes of K, of V are not needed any more.
template <int D, int NR, typename K, typename V, typename KD, typename VD, typename Vis>
__device__ __forceinline__ void stream_tile(StreamState<D, NR> &st, unsigned char *vhalf, K kfrag, V vfrag, KD k_done,
                                            VD v_done, bool masked, Vis vis, float cs, int lane) {
    using Gm = Geo<D>;
    constexpr int C = Gm::kChunks;
    constexpr int NKS = D / 32, NDB = D / 16;
    const int g = lane >> 4, c = lane & 15;
    f32x4 s[4][NR];
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        #pragma unroll
        for (int nr = 0; nr < NR; ++nr) s[kb][nr] = f32x4{0.f, 0.f, 0.f, 0.f};
        #pragma unroll
        for (int t = 0; t < NKS; ++t) {
            const bf16x8 a = kfrag(kb, t);
            #pragma unroll
            for (int nr = 0; nr < NR; ++nr)
                s[kb][nr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, st.qf[nr][t], s[kb][nr], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);     // one key block's operands at a time in registers
    }
    // V of keys 32 kst .. + 31 to LDS, and its transposing reads; LDS keeps a wave's order, so
    // the second half may follow the first's reads into the same place
    // (chunk numbers differ in bits that the swizzle's XOR passes on, so one address each is
    // kept, and made opaque: otherwise every chunk's is, in registers that then spill)
    unsigned to = lds_addr(vhalf) + c * Gm::kRowBytes + (((NKS * g) ^ swz<C>(c % C)) << 4);
    unsigned from;
    {
        const int key = 4 * g + (c >> 2);
        from = lds_addr(vhalf) + key * Gm::kRowBytes + ((((c & 3) >> 1) ^ swz<C>(key % C)) << 4) + (c & 1) * 8;
    }
    tie(to);
    tie(from);
    u32x2 v[NDB][2];
    auto store_v = [&](int kst) {
        #pragma unroll
        for (int r = 0; r < 2; ++r)
            #pragma unroll
            for (int t = 0; t < NKS; ++t) {
                const bf16x8 x = vfrag(2 * kst + r, t);
                asm volatile("ds_write_b128 %0, %1 offset:%2"
                             ::"v"(to ^ (t << 4)), "v"(__builtin_bit_cast(u32x4, x)), "i"(r * 16 * Gm::kRowBytes)
                             : "memory");
            }
    };
    auto read_v = [&]() {
        #pragma unroll
        for (int db = 0; db < NDB; ++db)
            #pragma unroll
            for (int r = 0; r < 2; ++r) {
                // key 16 r + 4 g + (c >> 2) has the swizzle of 4 g + (c >> 2) up to a multiple of C
                const unsigned at = from ^ ((unsigned)((2 * db) ^ swz<C>((16 * r) % C)) << 4);
                asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2"
                             : "=v"(v[db][r]) : "v"(at), "i"(r * 16 * Gm::kRowBytes) : "memory");
            }
    };
    k_done();
    __builtin_amdgcn_sched_barrier(0);
    store_v(0);
    read_v();
    store_v(1);
    v_done();
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 pb[NR][2];
    #pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        if (masked) {
            const unsigned long long x = vis(nr) >> (4 * g);
            const unsigned half[2] = {(unsigned)x, (unsigned)(x >> 32)};
            #pragma unroll
            for (int kb = 0; kb < 4; ++kb)
                #pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[kb][nr][i] = (half[kb >> 1] >> ((kb & 1) * 16 + i)) & 1u ? s[kb][nr][i] : kNegInf;
        }
        float mt = kNegInf;
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb)
            mt = fmaxf(mt, fmaxf(fmaxf(s[kb][nr][0], s[kb][nr][1]), fmaxf(s[kb][nr][2], s[kb][nr][3])));
        mt = rows_max(mt);
        const bool raise = mt * cs > st.m_run[nr] * cs + kRescaleSlack;
        if (__any(raise)) {
            const float m_new = raise ? mt : st.m_run[nr];
            const float alpha =
                (st.m_run[nr] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f((st.m_run[nr] - m_new) * cs);
            st.l_run[nr] *= alpha;
            #pragma unroll
            for (int db = 0; db < NDB; ++db)
                #pragma unroll
                for (int i = 0; i < 4; ++i) st.o[nr][db][i] *= alpha;
            st.m_run[nr] = m_new;
        }
        const float msc = (st.m_run[nr] == kNegInf) ? 0.f : st.m_run[nr] * cs;
        float sum = 0.f;
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb)
            #pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][nr][i], cs, -msc));
                sum += x;
                pb[nr][kb >> 1][(kb & 1) * 4 + i] = (__bf16)x;
            }
        st.l_run[nr] += sum;
    }
    #pragma unroll
    for (int kst = 0; kst < 2; ++kst) {
        if (kst == 1) {
            __builtin_amdgcn_sched_barrier(0);     // into the registers that the first half leaves
            read_v();
        }
        lds_wait<0>();
        #pragma unroll
        for (int db = 0; db < NDB; ++db) {
            tie(v[db][0]);
            tie(v[db][1]);
        }
        #pragma unroll
        for (int db = 0; db < NDB; ++db) {
            const u32x4 a = {v[db][0][0], v[db][0][1], v[db][1][0], v[db][1][1]};
            #pragma unroll
            for (int nr = 0; nr < NR; ++nr)
                st.o[nr][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pb[nr][kst],
                                                                       st.o[nr][db], 0, 0, 0);
        }
    }
}

template <int D, int NR, bool SMALL>
__global__ __launch_bounds__(kStreamWaves * kWave, kStreamWgPerCu) void kv4_stream_kernel(Kv4AttnParams p) {
    using Gm = Geo<D>;
    constexpr int NW = kStreamWaves, NT = NW * kWave;
    constexpr int R = 16 * NR;
    constexpr int NKS = D / 32, NDB = D / 16;
    static_assert(NW * 16 * D * 4 <= (int)sizeof(g_half), "the waves' results of a row tile fit their half tiles");

    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    const int wave_u = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int g4 = lane >> 4, c = lane & 15;
    const int w = xcd_contiguous_id(blockIdx.x, p.num_wg);
    unsigned char *vhalf = g_half + wave_u * (Gm::kTileBytes / 2);

    build_cumulative(p, [&](int L, int nodes) { return sequence_tiles(p, L, nodes); });

    const Shares sh(g_cum[p.B], p.num_wg);
    const int start = sh.start_of(w), end = sh.start_of(w + 1);

    int pos = start;
    int anc_b = -1;
    if (start >= end && tid == 0) p.ws_desc[w * 4] = -1;
    while (pos < end) {
        Piece pc;
        if (!next_piece(p, sh, w, start, end, pos, pc)) continue;
        const int b = pc.b, g = pc.g, rb = pc.rb, nodes = pc.nodes, rows_b = pc.rows_b, ntp = pc.ntp;

        if (needs_paths(p, pc) && anc_b != b) {
            if (wave_u == 0) {
                if (p.N <= kWave)
                    build_ancestor_masks_wave(p, lane < p.N ? p.parent[(size_t)b * p.N + lane] : -1);
                else
                    build_ancestor_masks_wave_lds(p, b);
            }
            anc_b = b;
            __syncthreads();
        }

        // ---- the query rows: a row past the unit's last one loads the unit's first
        StreamState<D, NR> st;
        int node[NR];
        #pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int at = rb * R + 16 * nr + c, row = at < rows_b ? at : rb * R;
            node[nr] = node_of(p, row);
            const uint16_t *qp = p.q + (((size_t)b * p.N + node[nr]) * p.Hq + g * p.G + row - node[nr] * p.G) * D;
            #pragma unroll
            for (int i = 0; i < NKS; ++i)
                st.qf[nr][i] = *reinterpret_cast<const bf16x8 *>(qp + g4 * (D / 4) + 8 * i);
            #pragma unroll
            for (int db = 0; db < NDB; ++db) st.o[nr][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            st.m_run[nr] = kNegInf;
            st.l_run[nr] = 0.f;
        }

        // ---- this wave's tiles; behind the last one its loads are repeated
        const int tp_end = min(pc.t_end, ntp);
        auto base_of = [&](int t) { return pc.real(min(t, tp_end - 1)) * KT; };
        int t = pc.t0 + wave_u;
        if (t < tp_end) {
            Raw4<D> raw;
            long long row[4];
            find_rows<SMALL>(p, pc, base_of(t), c, row);
            load_part<D, SMALL>(p, row, false, lane, raw.k, raw.ks);
            load_part<D, SMALL>(p, row, true, lane, raw.v, raw.vs);
            for (; t < tp_end; t += NW) {
                const int base = base_of(t);
                find_rows<SMALL>(p, pc, base_of(t + NW), c, row);
                if (base + KT > pc.L || (base < pc.sp.lo && base + KT > pc.sp.sinks)) drop_unseen<D>(pc, base, c, raw);
                stream_tile<D, NR>(
                    st, vhalf, [&](int kb, int i) { return from4x8(raw.k[kb][i], scale4(raw.ks[kb])); },
                    [&](int kb, int i) { return from4x8(raw.v[kb][i], scale4(raw.vs[kb])); },
                    [&]() { load_part<D, SMALL>(p, row, false, lane, raw.k, raw.ks); },
                    [&]() { load_part<D, SMALL>(p, row, true, lane, raw.v, raw.vs); },
                    base + KT > pc.L || !window_clear(pc.sp, base, p.N),
                    [&](int nr) { return prefix_bits(p, pc, base, node[nr]); }, p.scale_log2, lane);
            }
        }
        for (; t < pc.t_end; t += NW) {
            // tree rows, in bf16; a slot past the sequence's nodes reads node 0's row
            int ln = lane;
            tie(ln);                       // addresses are made here, not kept through the loop above
            const int j0 = (t - ntp) * KT + (ln & 15);
            auto tree_row = [&](const uint16_t *from, int kb, int i) {
                const int j = j0 + 16 * kb;
                return *reinterpret_cast<const bf16x8 *>(
                    from + (((size_t)b * p.N + (j < nodes ? j : 0)) * p.Hkv + g) * D + (ln >> 4) * (D / 4) + 8 * i);
            };
            stream_tile<D, NR>(
                st, vhalf, [&](int kb, int i) { return tree_row(p.k_tree, kb, i); },
                [&](int kb, int i) { return tree_row(p.v_tree, kb, i); }, []() {}, []() {}, true,
                [&](int nr) { return window_path(g_anc[node[nr]], t - ntp, pc.L, p); }, p.scale_log2, lane);
        }

        // ---- the waves' (max, sum, O^T) of a row tile meet in LDS and combine with the
        // log-sum-exp rule; thread (row, 8-column chunk) writes one 16-byte piece of the row
        constexpr int kCh = D / 8;
        float *ow = reinterpret_cast<float *>(g_half);                     // [NW][16][D]
        const float cs = p.scale_log2;
        int th = tid;
        tie(th);
        const int oc = th & 15, og = (th >> 4) & 3;
        #pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int first = rb * R + 16 * nr;
            if (nr > 0 && first >= rows_b) break;
            __syncthreads();               // half tiles, or the row tile before, have been read
            const float lw = rows_sum(st.l_run[nr]);
            #pragma unroll
            for (int db = 0; db < NDB; ++db)
                *reinterpret_cast<f32x4 *>(ow + (wave_u * 16 + oc) * D + db * 16 + 4 * og) = st.o[nr][db];
            if (og == 0) {
                g_ml[wave_u][oc][0] = st.m_run[nr];
                g_ml[wave_u][oc][1] = lw;
            }
            __syncthreads();
            for (int task = th; task < 16 * kCh; task += NT) {
                const int r = task / kCh, ch = task % kCh;
                if (first + r >= rows_b) continue;
                float M = kNegInf;
                #pragma unroll
                for (int u = 0; u < NW; ++u) M = fmaxf(M, g_ml[u][r][0]);
                float lsum = 0.f;
                float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int u = 0; u < NW; ++u) {
                    const float mu = g_ml[u][r][0];                // -inf: the wave saw nothing, or NaN only
                    const float sc = mu == kNegInf ? 0.f : __builtin_amdgcn_exp2f((mu - M) * cs);
                    lsum += sc * g_ml[u][r][1];
                    const f32x4 a0 = *reinterpret_cast<const f32x4 *>(ow + (u * 16 + r) * D + ch * 8);
                    const f32x4 a1 = *reinterpret_cast<const f32x4 *>(ow + (u * 16 + r) * D + ch * 8 + 4);
                    #pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[e] += sc * a0[e];
                        acc[4 + e] += sc * a1[e];
                    }
                }
                const float inv = 1.f / lsum;
                if (pc.complete) {
                    bf16x8 o;
                    #pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = (__bf16)(acc[e] * inv);
                    const int nd = node_of(p, first + r), h = g * p.G + first + r - nd * p.G;
                    *reinterpret_cast<bf16x8 *>(p.out + (((size_t)b * p.N + nd) * p.Hq + h) * D + ch * 8) = o;
                    if (ch == 0 && p.lse)
                        p.lse[((size_t)b * p.N + nd) * p.Hq + h] = M * p.scale + __builtin_amdgcn_logf(lsum) * kLn2;
                } else {
                    // a piece: normalised by its own sum, fp16 times a power of two (a piece may
                    // hold no key that the row sees, and is left out by the joining kernel then)
                    const bool none = lsum == 0.f;
                    const float top = row_top(
                        [&](auto take) {
                            #pragma unroll
                            for (int e = 0; e < 8; ++e) take(acc[e]);
                        },
                        [&](float x) {
                            #pragma unroll
                            for (int o = 1; o < kCh; o <<= 1) x = fmaxf(x, __shfl_xor(x, o));
                            return x;
                        });
                    float unscale;
                    const float scaled = none ? 0.f : inv * part_scale(top * inv, unscale);
                    f16x8 f;
                    #pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = (_Float16)(acc[e] * scaled);
                    const size_t at = (size_t)pc.slot * p.rows_per_block + 16 * nr + r;
                    *reinterpret_cast<f16x8 *>(p.ws_o + at * D + ch * 8) = f;
                    if (ch == 0)
                        *reinterpret_cast<f32x4 *>(p.ws_ml + at * 4) =
                            f32x4{part_max(M, lsum, cs), lsum, none ? 1.f : unscale, 0.f};
                }
            }
        }
        __syncthreads();                   // the next piece's half tiles and ancestor sets
    }

    clear_padding<D, NT>(p, w);
}

template <int D>
hipError_t launch_d(const Kv4AttnParams &p, hipStream_t s) {
    auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(p.num_wg), dim3(kStreamWaves * kWave), s, p); };
    hipError_t e;
    switch (p.rows_per_block) {
        case 16: e = p.P < 16 ? go(kv4_stream_kernel<D, 1, true>) : go(kv4_stream_kernel<D, 1, false>); break;
        case 32: e = p.P < 16 ? go(kv4_stream_kernel<D, 2, true>) : go(kv4_stream_kernel<D, 2, false>); break;
        default: e = launch_kv4_wide(p, D, s);
    }
    if (e != hipSuccess || p.num_wg == 1) return e;
    constexpr int kRowsPerWg = 256 / (D / 8);
    const int chunks = (p.rows_per_block + kRowsPerWg - 1) / kRowsPerWg;
    const int stride = (p.num_wg + kNumXcd - 1) / kNumXcd * kNumXcd;
    return launch_kernel(tree_attention_merge_fine_kernel<D>, dim3(stride * chunks), dim3(256), s,
                         static_cast<const AttnParams &>(p), stride);
}

}  // namespace

hipError_t launch_kv4_attention(const Kv4AttnParams &p, int head_dim, hipStream_t s) {
    if (head_dim == 64) return launch_d<64>(p, s);
    if (head_dim == 128) return launch_d<128>(p, s);
    return hipErrorInvalidValue;
}

}  // namespace tv
