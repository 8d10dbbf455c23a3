// Tree-masked attention over a paged prefix held in 4 bits (kv4.h), with an optional
// sliding window, for gfx950.
//
// The function is tree_verify_attention's, with the values that the codes stand for in
// place of the cache's rows. A key of a KV head is D/2 bytes of codes and D/32 scale bytes
// for K and the same for V, 136 bytes at head size 128 where bf16 takes 512.
//
// Work decomposition: units (sequence, KV head, block of 16 NR query rows), their 64-key
// tiles laid end to end and shared out equally over the workgroups as in
// tree_attention.hip. Within a piece the workgroup's waves take its tiles in turn, each by
// itself: no barrier until the piece ends, where the waves' (max, sum, O) meet in LDS.
//
// One tile of one wave, v_mfma_f32_16x16x32_bf16 throughout. Lane l = 16 g + c:
//   S^T = K Q^T: the lane holds key 16 kb + c of every key block kb, and of it the D/4
//     values from (D/4) g on, which are one load of 16 (8) bytes of codes. That order of
//     the head dimension is not the operand's own, but the sum over it is the same in any
//     order, so Q's fragments are loaded in the same one and K needs no shuffle: eight
//     codes become one operand by four conversions.
//   O^T += V^T P^T: the operand wants eight keys of one column per lane. The lane
//     converts the same part of V's row and stores it to a row-major tile of the wave's
//     own in LDS (16-byte chunks swizzled by the key), and ds_read_b64_tr_b16 reads it
//     transposed, with the key order that the scores' accumulators have.
// The codes of a wave's next tile are on their way in registers while it computes one.
#include "tree_attention_kv4.h"

namespace tv {
namespace {

// A wave's raw loads of one prefix tile.
template <int D>
struct Raw4 {
    static constexpr int W = D / 32;                   // dwords of codes per lane and key
    unsigned k[4][W], v[4][W];
    unsigned ks[4], vs[4];                             // scale bytes
    unsigned live;                                     // bit kb: the lane's key of block kb counts
};

template <int D, int NR>
struct StreamState {
    static constexpr int NKS = D / 32;                 // k-steps over the head dim (S)
    static constexpr int NDB = D / 16;                 // 16-wide head-dim blocks of O^T
    bf16x8 qf[NR][NKS];
    f32x4 o[NR][NDB];
    float m_run[NR], l_run[NR];
};

// Page ids of the lane's keys of the prefix tile at position `base`.
__device__ __forceinline__ void load_ids(const Kv4AttnParams &p, int b, int base, int c, int (&ids)[4]) {
    const int32_t *row = p.page_table + (size_t)b * p.max_pages;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) ids[kb] = row[min((base + 16 * kb + c) >> p.p_shift, p.max_pages - 1)];
}

// Their codes and scales. A key that no node sees reads the cache's first row, and counts
// as zeros.
template <int D>
__device__ __forceinline__ void load_raw(const Kv4AttnParams &p, const Piece &pc, int base, int lane, const int (&ids)[4],
                                         Raw4<D> &r) {
    const int c = lane & 15, g = lane >> 4;
    r.live = 0;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        const long long at = row_of(p, pc.g, base + 16 * kb + c, ids[kb], pc.L, pc.sp), row = max(at, 0ll);
        r.live |= (unsigned)(at >= 0) << kb;
        load_dwords(r.k[kb], p.k4 + row * (D / 2) + g * (D / 8));
        load_dwords(r.v[kb], p.v4 + row * (D / 2) + g * (D / 8));
        const uint8_t *s = p.scales + row * (D / 16) + (g * (D / 4)) / kBlock4;
        r.ks[kb] = s[0];
        r.vs[kb] = s[D / kBlock4];
    }
}

template <int D>
__device__ __forceinline__ void drop_dead(Raw4<D> &r) {
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb)
        if (!((r.live >> kb) & 1u)) {
            #pragma unroll
            for (int w = 0; w < Raw4<D>::W; ++w) r.k[kb][w] = r.v[kb][w] = 0;
            r.ks[kb] = r.vs[kb] = 127;
        }
}

// One tile: kfrag(kb, t) and vfrag(kb, t) give eight values of the lane's key of block kb,
// from head-dim index (D/4) g + 8 t on; `vis` the keys that the lane's row of tile nr sees.
template <int D, int NR, typename K, typename V, typename Vis>
__device__ __forceinline__ void stream_tile(StreamState<D, NR> &st, unsigned char *vtile, K kfrag, V vfrag,
                                            bool masked, Vis vis, float cs, int lane) {
    using Gm = Geo<D>;
    constexpr int C = Gm::kChunks;
    constexpr int NKS = D / 32, NDB = D / 16;
    const int g = lane >> 4, c = lane & 15;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb)
        #pragma unroll
        for (int t = 0; t < NKS; ++t) {
            const int key = 16 * kb + c;
            *reinterpret_cast<bf16x8 *>(vtile + key * Gm::kRowBytes + (((NKS * g + t) ^ swz<C>(key % C)) << 4)) =
                vfrag(kb, t);
        }
    f32x4 s[NR][4];
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        #pragma unroll
        for (int nr = 0; nr < NR; ++nr) s[nr][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
        #pragma unroll
        for (int t = 0; t < NKS; ++t) {
            const bf16x8 a = kfrag(kb, t);
            #pragma unroll
            for (int nr = 0; nr < NR; ++nr)
                s[nr][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, st.qf[nr][t], s[nr][kb], 0, 0, 0);
        }
    }
    bf16x8 pb[NR][2];
    #pragma unroll
    for (int nr = 0; nr < NR; ++nr) {
        if (masked) {
            const unsigned long long x = vis(nr);
            #pragma unroll
            for (int kb = 0; kb < 4; ++kb)
                #pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[nr][kb][i] = ((x >> (kb * 16 + 4 * g + i)) & 1ull) ? s[nr][kb][i] : kNegInf;
        }
        float mt = kNegInf;
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb)
            mt = fmaxf(mt, fmaxf(fmaxf(s[nr][kb][0], s[nr][kb][1]), fmaxf(s[nr][kb][2], s[nr][kb][3])));
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
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[nr][kb][i], cs, -msc));
                sum += x;
                pb[nr][kb >> 1][(kb & 1) * 4 + i] = (__bf16)x;
            }
        st.l_run[nr] += sum;
    }
    // the transposing reads of half a tile at a time, the second half's in flight during
    // the first half's products
    const unsigned vbase = lds_addr(vtile);
    u32x2 v[2][NDB][2];
    auto read_v = [&](int kst) {
        #pragma unroll
        for (int db = 0; db < NDB; ++db)
            #pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int key = (2 * kst + r) * 16 + 4 * g + (c >> 2);
                const int chunk = 2 * db + ((c & 3) >> 1);
                const unsigned addr =
                    vbase + key * Gm::kRowBytes + ((unsigned)(chunk ^ swz<C>(key % C)) << 4) + (c & 1) * 8;
                asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(v[kst][db][r]) : "v"(addr) : "memory");
            }
    };
    read_v(0);
    #pragma unroll
    for (int kst = 0; kst < 2; ++kst) {
        lds_wait<0>();
        #pragma unroll
        for (int db = 0; db < NDB; ++db) {
            tie(v[kst][db][0]);
            tie(v[kst][db][1]);
        }
        if (kst == 0) read_v(1);
        #pragma unroll
        for (int db = 0; db < NDB; ++db) {
            const u32x4 a = {v[kst][db][0][0], v[kst][db][0][1], v[kst][db][1][0], v[kst][db][1][1]};
            #pragma unroll
            for (int nr = 0; nr < NR; ++nr)
                st.o[nr][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pb[nr][kst],
                                                                       st.o[nr][db], 0, 0, 0);
        }
    }
}

template <int D, int NW, int NR>
__global__ __launch_bounds__(NW * kWave) void kv4_stream_kernel(Kv4AttnParams p) {
    using Gm = Geo<D>;
    constexpr int NT = NW * kWave;
    constexpr int R = 16 * NR;
    constexpr int NKS = D / 32, NDB = D / 16;
    static_assert(NW * Gm::kTileBytes <= (int)sizeof(g_ring) && NW * R * D * 4 <= (int)sizeof(g_ring) &&
                      NW * R * 8 <= (int)sizeof(g_anc_alt),
                  "the waves' V tiles, and their results, fit the ring");

    const int tid = threadIdx.x;
    const int lane = tid & (kWave - 1);
    const int wave_u = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int g4 = lane >> 4, c = lane & 15;
    const int w = xcd_contiguous_id(blockIdx.x, p.num_wg);
    unsigned char *vtile = g_ring + wave_u * Gm::kTileBytes;

    build_cumulative<NT>(p);

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
            const int row = rb * R + 16 * nr + c, qrow = row < rows_b ? row : rb * R;
            node[nr] = node_of(p, qrow);
            const uint16_t *qp =
                p.q + (((size_t)b * p.N + node[nr]) * p.Hq + g * p.G + qrow - node[nr] * p.G) * D + g4 * (D / 4);
            #pragma unroll
            for (int t = 0; t < NKS; ++t)
                st.qf[nr][t] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8 *>(qp + 8 * t));
            #pragma unroll
            for (int db = 0; db < NDB; ++db) st.o[nr][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            st.m_run[nr] = kNegInf;
            st.l_run[nr] = 0.f;
        }

        // ---- this wave's tiles
        const int tp_end = min(pc.t_end, ntp);
        auto base_of = [&](int t) { return pc.real(t) * KT; };
        Raw4<D> raw;
        int ids[4];
        int t = pc.t0 + wave_u;
        if (t < tp_end) {
            load_ids(p, b, base_of(t), c, ids);
            load_raw<D>(p, pc, base_of(t), lane, ids, raw);
            if (t + NW < tp_end) load_ids(p, b, base_of(t + NW), c, ids);
        }
        for (; t < tp_end; t += NW) {
            const int base = base_of(t);
            Raw4<D> cur = raw;
            if (t + NW < tp_end) {
                load_raw<D>(p, pc, base_of(t + NW), lane, ids, raw);
                if (t + 2 * NW < tp_end) load_ids(p, b, base_of(t + 2 * NW), c, ids);
            }
            const bool masked = base + KT > pc.L || !window_clear(pc.sp, base, p.N);
            if (__any(cur.live != 15u)) drop_dead(cur);
            stream_tile<D, NR>(
                st, vtile, [&](int kb, int i) { return from4x8(cur.k[kb][i], scale4(cur.ks[kb])); },
                [&](int kb, int i) { return from4x8(cur.v[kb][i], scale4(cur.vs[kb])); }, masked,
                [&](int nr) { return prefix_bits(p, pc, base, node[nr]); }, p.scale_log2, lane);
        }
        for (; t < pc.t_end; t += NW) {
            // tree rows, in bf16; a slot past the sequence's nodes reads node 0's row
            const int j0 = (t - ntp) * KT;
            auto tree_row = [&](const uint16_t *from, int kb, int i) {
                const int j = j0 + 16 * kb + c;
                return *reinterpret_cast<const bf16x8 *>(
                    from + (((size_t)b * p.N + (j < nodes ? j : 0)) * p.Hkv + g) * D + g4 * (D / 4) + 8 * i);
            };
            stream_tile<D, NR>(
                st, vtile, [&](int kb, int i) { return tree_row(p.k_tree, kb, i); },
                [&](int kb, int i) { return tree_row(p.v_tree, kb, i); }, true,
                [&](int nr) { return window_path(g_anc[node[nr]], t - ntp, pc.L, p); }, p.scale_log2, lane);
        }

        // ---- the waves' (max, sum, O^T) meet in LDS and combine with the log-sum-exp rule;
        // thread (row, 8-column chunk) writes one 16-byte piece of the row
        constexpr int kCh = D / 8;
        float *ow = reinterpret_cast<float *>(g_ring);                     // [NW][R][D]
        float *mlw = reinterpret_cast<float *>(g_anc_alt);                 // [NW][R][2]
        __syncthreads();
        #pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int r = wave_u * R + 16 * nr + c;
            const float lw = rows_sum(st.l_run[nr]);
            #pragma unroll
            for (int db = 0; db < NDB; ++db)
                *reinterpret_cast<f32x4 *>(ow + (size_t)r * D + db * 16 + 4 * g4) = st.o[nr][db];
            if (g4 == 0) {
                mlw[r * 2] = st.m_run[nr];
                mlw[r * 2 + 1] = lw;
            }
        }
        __syncthreads();
        const int nrows = min(R, rows_b - rb * R);
        const float cs = p.scale_log2;
        for (int task = tid; task < R * kCh; task += NT) {
            const int r = task / kCh, ch = task % kCh;
            if (r >= nrows) continue;
            float M = kNegInf;
            #pragma unroll
            for (int u = 0; u < NW; ++u) M = fmaxf(M, mlw[(u * R + r) * 2]);
            float lsum = 0.f;
            float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            #pragma unroll
            for (int u = 0; u < NW; ++u) {
                const float mu = mlw[(u * R + r) * 2];
                if (mu == kNegInf) continue;                       // the wave saw nothing
                const float sc = __builtin_amdgcn_exp2f((mu - M) * cs);
                lsum += sc * mlw[(u * R + r) * 2 + 1];
                const f32x4 a0 = *reinterpret_cast<const f32x4 *>(ow + ((size_t)u * R + r) * D + ch * 8);
                const f32x4 a1 = *reinterpret_cast<const f32x4 *>(ow + ((size_t)u * R + r) * D + ch * 8 + 4);
                #pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[e] += sc * a0[e];
                    acc[4 + e] += sc * a1[e];
                }
            }
            const float inv = 1.f / lsum;
            const int ur = rb * R + r;
            if (pc.complete) {
                bf16x8 o;
                #pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (__bf16)(acc[e] * inv);
                const int nd = node_of(p, ur), h = g * p.G + ur - nd * p.G;
                *reinterpret_cast<bf16x8 *>(p.out + (((size_t)b * p.N + nd) * p.Hq + h) * D + ch * 8) = o;
                if (ch == 0 && p.lse)
                    p.lse[((size_t)b * p.N + nd) * p.Hq + h] = M * p.scale + __builtin_amdgcn_logf(lsum) * kLn2;
            } else {
                // a piece: normalised by its own sum, fp16 times a power of two (a piece may
                // hold no key that the row sees: max -inf, left out by the joining kernel)
                const bool none = M == kNegInf;
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
                *reinterpret_cast<f16x8 *>(p.ws_o + ((size_t)pc.slot * p.rows_per_block + r) * D + ch * 8) = f;
                if (ch == 0)
                    *reinterpret_cast<f32x4 *>(p.ws_ml + ((size_t)pc.slot * p.rows_per_block + r) * 4) =
                        f32x4{none ? kNegInf : M * cs, none ? 0.f : lsum, none ? 1.f : unscale, 0.f};
            }
        }
        __syncthreads();                   // the next piece's V tiles and ancestor sets
    }

    clear_padding<D, NT>(p, w);
}

template <int D>
hipError_t launch_d(const Kv4AttnParams &p, hipStream_t s) {
    auto go = [&](auto kernel, int waves) { return launch_kernel(kernel, dim3(p.num_wg), dim3(waves * kWave), s, p); };
    hipError_t e;
    switch (p.rows_per_block) {
        case 16: e = go(kv4_stream_kernel<D, 8, 1>, 8); break;
        case 32: e = go(kv4_stream_kernel<D, 8, 2>, 8); break;
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
