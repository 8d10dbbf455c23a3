// What each sequence of a batch with shared prefixes has behind the shared
// tiles, where it has at most 48 query rows per KV head: a part of
// tree_attention_shared.hip, whose ring, tables and helpers it uses.
//
// A unit is one (sequence, KV head): its keys are the prefix positions behind
// the shared tiles and then its tree nodes, one list without a gap, in tiles
// of 8 KB of keys and 8 KB of values (32 keys of head size 128, 64 of 64). All
// units' tiles are laid end to end (kOwnTile places each, and one for the start
// of a unit) and every wave takes those that begin in its equal share of the
// places, by itself: it has 16 KB of the ring to itself, loads a tile into it, and
// computes all RT x 16 rows of the unit on it with v_mfma_f32_16x16x32_bf16 in the
// layout of the narrow units (narrow_tile). The next tile's keys are loaded once
// this tile's scores are taken, its values once this tile's have been used, also
// across units; nothing is shared between waves, so there is no barrier, and a
// unit that ends costs the other waves nothing. The eight waves keep up to 128 KB
// in flight per CU, which bounds the kernel by the stream of K and V.
//
// Against row blocks for the own units too, us per call: decoding 64 sequences (own
// keys 16-512 behind 4096 shared ones) 54 and 35, 12-token trees of 16 sequences with
// 32 KV heads 74 and 48; from 64 rows on the row blocks are ahead (67 and 50).
#pragma once

namespace tv {
namespace {

// A tile of a wave's share (wave-uniform). `base` is the place of its unit, whose
// tile ti begins at base + 1 + ti * kOwnTile; from, L, nodes: of its sequence.
struct OwnTile {
    int b, g, ti, nt, base;
    int from, L, nodes;
    bool ok;
};

// LDS reads with their wait in one block: no register that is still being read can
// be spilled or moved in between. The memory clobber keeps them behind the tile's
// loads' wait and ahead of the loads that refill the tile. OFF: bytes behind each address.
template <int OFF>
__device__ __forceinline__ void lds_read4(u32x4 (&a)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3) {
    asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\t"
                 "ds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "i"(OFF) : "memory");
}
template <int OFF>
__device__ __forceinline__ void lds_read2(u32x4 (&a)[2], unsigned a0, unsigned a1) {
    asm volatile("ds_read_b128 %0, %2 offset:%4\n\tds_read_b128 %1, %3 offset:%4\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a[0]), "=&v"(a[1]) : "v"(a0), "v"(a1), "i"(OFF) : "memory");
}
// Transposing reads at four addresses, and OFF2 bytes from each.
template <int OFF, int OFF2>
__device__ __forceinline__ void lds_read_tr8(u32x2 (&v)[4][2], unsigned a0, unsigned a1, unsigned a2,
                                             unsigned a3) {
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(v[0][0]), "=&v"(v[0][1]), "=&v"(v[1][0]), "=&v"(v[1][1]), "=&v"(v[2][0]), "=&v"(v[2][1]),
                   "=&v"(v[3][0]), "=&v"(v[3][1])
                 : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "i"(OFF), "i"(OFF + OFF2) : "memory");
}
// The compiler keeps what depends on x in the loop instead of holding it across.
__device__ __forceinline__ unsigned here(unsigned x) {
    asm volatile("" : "+v"(x));
    return x;
}

template <int... I, typename F>
__device__ __forceinline__ void static_for_of(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>{}), ...);
}
// f(0) .. f(N - 1) with constants.
template <int N, typename F>
__device__ __forceinline__ void static_for(F f) {
    static_for_of(std::make_integer_sequence<int, N>{}, f);
}

template <int D, int RT>
struct OwnState {
    static constexpr int NKS = D / 32, NDB = D / 16;
    bf16x8 q[RT][NKS];
    f32x4 o[RT][NDB];
    float m[RT], l[RT];
};

// Wave `wid` of `waves`: its share of the own units' tiles.
template <int D, int RT>
__device__ __forceinline__ void own_shares(const SharedAttnParams &p, int wid, int waves) {
    using Og = OwnGeo<D>;
    constexpr int C = Geo<D>::kChunks, RB = Geo<D>::kRowBytes;
    constexpr int NKS = D / 32, NDB = D / 16, KN = Og::kKeys, NKB = KN / 16, NST = KN / 32;
    constexpr int NL = Og::kLoads, KPL = Og::kKeysPerLoad;
    constexpr bool kAhead = RT == 1;                   // the next unit's queries fit beside this one's
    const int lane = threadIdx.x & (kWave - 1), g4 = lane >> 4, i16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    auto uni = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    const int first = uni(g_vcum[p.groups]), total = uni(g_vcum[p.groups + p.B]) - first;
    // every share is so long that a tile begins in it: the pieces of a split unit sit in
    // consecutive waves
    waves = min(waves, total / (kOwnTile + 1));
    if (wid >= waves) return;
    const int start = uni(first + (int)((long long)wid * total / waves));
    const int end = uni(first + (int)((long long)(wid + 1) * total / waves));

    unsigned char *ring = g_ring + wave * 2 * Og::kHalfBytes;
    const unsigned kbase = lds_addr(ring), vbase = kbase + Og::kHalfBytes;
    const size_t row_bytes = (size_t)p.Hkv * RB;
    const int mask = p.P - 1;
    const float c = p.scale_log2;
    // this lane's rows: node and head of the group
    int rnode[RT], rhead[RT];
    #pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        rnode[rt] = (rt * 16 + i16) / p.G;
        rhead[rt] = rt * 16 + i16 - rnode[rt] * p.G;
    }

    // ---- the share's tiles, one after another
    auto look_up = [&](OwnTile &t) {
        t.from = uni(shared_tiles_of(t.b)) * KT;
        t.L = uni(g_slen[t.b]);
        t.nodes = uni(g_ncum[t.b + 1] - g_ncum[t.b]);
        t.nt = own_tiles<D>(t.L, t.from, t.nodes);
    };
    auto next = [&](OwnTile t) {
        if (t.ti + 1 < t.nt) {
            ++t.ti;
        } else {
            t.base += t.nt * kOwnTile + 1;
            t.ti = 0;
            if (++t.g == p.Hkv) {
                t.g = 0;
                do {                                   // the next sequence that has nodes
                    if (++t.b == p.B) {
                        t.ok = false;
                        return t;
                    }
                    look_up(t);
                } while (t.nt == 0);
            }
        }
        t.ok = t.base + 1 + t.ti * kOwnTile < end;
        return t;
    };
    OwnTile cur;
    {
        int lo = 0, hi = p.B - 1;                      // the sequence that holds place `start`
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (g_vcum[p.groups + mid] <= start) lo = mid; else hi = mid - 1;
        }
        cur.b = uni(lo);
        look_up(cur);
        const int off = start - uni(g_vcum[p.groups + cur.b]);
        const int per = cur.nt * kOwnTile + 1;
        cur.g = uni(off / per);
        cur.base = start - (off - cur.g * per);
        cur.ti = (max(start - cur.base - 1, 0) + kOwnTile - 1) / kOwnTile;     // the first that begins here
        cur.ok = cur.base + 1 + cur.ti * kOwnTile < end;
        if (cur.ti == cur.nt) {                        // all of this unit's began before: the next one's first
            cur.ti = cur.nt - 1;
            cur = next(cur);
        }
    }
    if (!cur.ok) return;

    // ---- loads. Lane l of load i brings 16 bytes of key i * KPL + l / C
    auto first_key = [&](const OwnTile &t) { return t.from + t.ti * KN; };
    auto fetch_ids = [&](const OwnTile &t) {           // page of key lane % KN
        const int x = first_key(t) + (lane & (KN - 1));
        return p.page_table[(size_t)t.b * p.max_pages + (max(min(x, t.L - 1), 0) >> p.p_shift)];
    };
    auto issue = [&](const OwnTile &t, int ids, bool is_v) {
        const int x0 = first_key(t);
        const char *cache = reinterpret_cast<const char *>((is_v ? p.v_cache : p.k_cache) + (size_t)t.g * D);
        const char *tree =
            reinterpret_cast<const char *>((is_v ? p.v_tree : p.k_tree) + ((size_t)t.b * p.N * p.Hkv + t.g) * D);
        unsigned char *dst = ring + (is_v ? Og::kHalfBytes : 0);
        const int l = (int)here((unsigned)lane);
        #pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int kk = i * KPL + l / C, x = x0 + kk, j = x - t.L;
            const int id = __shfl(ids, kk);
            // a key past the last one, or without a page, reads tree node 0 (finite)
            const bool cached = j < 0 && (unsigned)id < (unsigned)p.num_pages;
            const size_t row = cached ? ((size_t)(unsigned)id << p.p_shift) + (x & mask)
                                      : (size_t)(j >= 0 && j < t.nodes ? j : 0);
            const char *a = (cached ? cache : tree) + row * row_bytes + (((l % C) ^ swz<C>(kk % C)) << 4);
            __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)a, (LDS_AS void *)(dst + i * 1024), 16, 0, 0);
        }
    };
    auto load_q = [&](const OwnTile &t, bf16x8 (&q)[RT][NKS]) {
        const int rows = t.nodes * p.G;
        #pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const bool real = rt * 16 + i16 < rows;    // others take row 0 and are not stored
            const uint16_t *qp = p.q + (((size_t)t.b * p.N + (real ? rnode[rt] : 0)) * p.Hq + t.g * p.G +
                                        (real ? rhead[rt] : 0)) * D + g4 * 8;
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                q[rt][ks] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8 *>(qp + ks * 32));
        }
    };

    OwnState<D, RT> st;
    bf16x8 qn[kAhead ? RT : 1][NKS];
    // Ancestor sets of a sequence's tree (of 64 nodes at most): lane i holds node i's
    int anc_b = -1, par = -1, par_b = -1;
    unsigned long long anc = 0ull;
    auto build_anc = [&](int b, int nodes) {
        int j = lane < nodes && par >= 0 && par < lane ? par : -1;
        anc = lane < nodes ? 1ull << lane : 0ull;
        while (__any(j >= 0)) {
            const int src = j >= 0 ? j : lane;
            const unsigned lo = (unsigned)__shfl((int)(unsigned)anc, src);
            const unsigned hi = (unsigned)__shfl((int)(unsigned)(anc >> 32), src);
            const int jj = __shfl(j, src);
            if (j >= 0) {
                anc |= ((unsigned long long)hi << 32) | lo;
                j = jj;
            }
        }
        anc_b = b;
    };

    int piece_ti = cur.ti;                             // first tile of the piece that is being computed
    bool fresh = true;
    int ids = fetch_ids(cur);
    if constexpr (kAhead) load_q(cur, qn);
    issue(cur, ids, false);
    issue(cur, ids, true);
    OwnTile nxt = next(cur);
    int ids_after = 0;                                 // pages of the tile behind nxt
    if (nxt.ok) ids = fetch_ids(nxt);

    for (;;) {
        const int L = cur.L, nodes = cur.nodes;
        if (fresh) {                                   // a unit's (part's) first tile
            if constexpr (kAhead) {
                #pragma unroll
                for (int rt = 0; rt < RT; ++rt)
                    #pragma unroll
                    for (int ks = 0; ks < NKS; ++ks) st.q[rt][ks] = qn[rt][ks];
            } else {
                load_q(cur, st.q);
            }
            #pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                st.m[rt] = kNegInf;
                st.l[rt] = 0.f;
                #pragma unroll
                for (int db = 0; db < NDB; ++db) st.o[rt][db] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
            if (par_b != cur.b) {
                par = lane < nodes ? p.parent[(size_t)cur.b * p.N + lane] : -1;
                par_b = cur.b;
            }
            piece_ti = cur.ti;
            fresh = false;
        }
        // ---- scores and softmax, 16 rows at a time, as in the narrow units; everything issued
        // behind this tile's keys is its values
        wait_vmcnt<NL>();
        const int x0 = first_key(cur);
        u32x4 pb[RT][NST];
        if (x0 + KN > L && anc_b != cur.b) build_anc(cur.b, nodes);
        #pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            f32x4 s[NKB];
            // key kb * 16 + i16: its row, and its swizzle, are a constant from key i16's
            const unsigned ka = here(kbase + i16 * RB + ((unsigned)(g4 ^ swz<C>(i16 % C)) << 4));
            static_for<NKB>([&](auto kb_) {
                constexpr int kb = decltype(kb_)::value;
                u32x4 a[NKS];
                if constexpr (NKS == 4) lds_read4<kb * 16 * RB>(a, ka, ka ^ 64u, ka ^ 128u, ka ^ 192u);
                else lds_read2<kb * 16 * RB>(a, ka, ka ^ 64u);
                s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int ks = 0; ks < NKS; ++ks)
                    s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[ks]),
                                                                    st.q[rt][ks], s[kb], 0, 0, 0);
            });
            if (x0 + KN > L) {
                const int nd = rt * 16 + i16 < nodes * p.G ? rnode[rt] : 0;
                const unsigned lo = (unsigned)__shfl((int)(unsigned)anc, nd);
                const unsigned hi = (unsigned)__shfl((int)(unsigned)(anc >> 32), nd);
                unsigned long long vis = ((unsigned long long)hi << 32) | lo;
                vis = x0 >= L ? vis >> min(x0 - L, 63) : (vis << (L - x0)) | ((1ull << (L - x0)) - 1ull);
                #pragma unroll
                for (int kb = 0; kb < NKB; ++kb)
                    #pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[kb][i] = ((vis >> (kb * 16 + 4 * g4 + i)) & 1ull) ? s[kb][i] : kNegInf;
            }
            float mt = kNegInf;
            #pragma unroll
            for (int kb = 0; kb < NKB; ++kb)
                mt = fmaxf(mt, fmaxf(fmaxf(s[kb][0], s[kb][1]), fmaxf(s[kb][2], s[kb][3])));
            mt = rows_max(mt);
            const bool raise = mt * c > st.m[rt] * c + kRescaleSlack;
            if (__any(raise)) {
                const float m_new = raise ? mt : st.m[rt];
                const float alpha =
                    (st.m[rt] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f((st.m[rt] - m_new) * c);
                st.l[rt] *= alpha;
                #pragma unroll
                for (int db = 0; db < NDB; ++db)
                    #pragma unroll
                    for (int i = 0; i < 4; ++i) st.o[rt][db][i] *= alpha;
                st.m[rt] = m_new;
            }
            const float msc = (st.m[rt] == kNegInf) ? 0.f : st.m[rt] * c;
            float ps = 0.f;
            #pragma unroll
            for (int k = 0; k < NST; ++k) {
                bf16x8 x8;
                #pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * k + (e >> 2)][e & 3], c, -msc));
                    ps += x;
                    x8[e] = (__bf16)x;
                }
                pb[rt][k] = __builtin_bit_cast(u32x4, x8);
            }
            st.l[rt] += ps;
        }
        // the tile's keys have been read: the next one's may come
        OwnTile nn = nxt;
        if (nxt.ok) {
            nn = next(nxt);
            if (nn.ok) ids_after = fetch_ids(nn);
            if constexpr (kAhead) {
                if (nxt.b != cur.b || nxt.g != cur.g) load_q(nxt, qn);
            }
            issue(nxt, ids, false);
        }
        // ---- O^T += V^T P^T: behind this tile's values there are the next one's keys
        if (nxt.ok) wait_vmcnt<NL>();
        else wait_vmcnt<0>();
        const int vkey = 4 * g4 + (i16 >> 2);           // of the first key block
        const unsigned va = here(vbase + vkey * RB + ((unsigned)(((i16 & 3) >> 1) ^ swz<C>(vkey % C)) << 4) +
                                 (i16 & 1) * 8);
        static_for<NST * (NDB / 4)>([&](auto step) {
                constexpr int k = decltype(step)::value / (NDB / 4), d0 = decltype(step)::value % (NDB / 4) * 4;
                u32x2 v[4][2];
                lds_read_tr8<k * 32 * RB, 16 * RB>(v, va ^ (d0 + 0) * 32u, va ^ (d0 + 1) * 32u, va ^ (d0 + 2) * 32u,
                                                   va ^ (d0 + 3) * 32u);
                #pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const u32x4 av = {v[d][0][0], v[d][0][1], v[d][1][0], v[d][1][1]};
                    #pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
                        st.o[rt][d0 + d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, av), __builtin_bit_cast(bf16x8, pb[rt][k]),
                            st.o[rt][d0 + d], 0, 0, 0);
                }
        });
        // ---- the unit's (or the share's) last tile. A whole unit leaves its rows, in out if there
        // are no shared keys beside it; a piece goes to a slot of this wave, normalised by its own
        // sum: slot 0 continues a unit, slot 1 begins one
        const bool ends = cur.ti + 1 == cur.nt;
        if (ends || !nxt.ok) {
            const bool whole = piece_ti == 0 && ends, last = whole && cur.from == 0;
            const int slot = wid * 2 + (piece_ti > 0 ? 0 : 1);
            if (lane == 0) {
                int32_t *rec = p.ws_unit + 2 * (cur.b * p.Hkv + cur.g);
                if (piece_ti == 0) rec[0] = whole ? -1 : slot;
                if (ends) rec[1] = wid;
            }
            const size_t all = (size_t)p.B * p.N * p.Hq;
            #pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int r = rt * 16 + i16;
                const float l = rows_sum(st.l[rt]);
                const float inv = l > 0.f ? 1.f / l : 0.f;
                float unscale = 1.f, scaled = inv;
                if (!last) {
                    const float top = row_top(
                        [&](auto take) {
                            #pragma unroll
                            for (int db = 0; db < NDB; ++db)
                                #pragma unroll
                                for (int i = 0; i < 4; ++i) take(st.o[rt][db][i]);
                        },
                        rows_max);
                    scaled *= part_scale(top * inv, unscale);
                }
                if (r >= nodes * p.G) continue;
                const size_t row = ((size_t)cur.b * p.N + rnode[rt]) * p.Hq + cur.g * p.G + rhead[rt];
                const size_t piece = (size_t)slot * (RT * 16) + r;
                uint16_t *o = last ? p.out + row * D : whole ? p.ws_whole + (all + row) * D : p.own_o + piece * D;
                #pragma unroll
                for (int db = 0; db < NDB; ++db) {
                    bf16x4 v;
                    if (last) {
                        #pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = (__bf16)(st.o[rt][db][i] * inv);
                    } else {
                        f16x4 f;
                        #pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = (_Float16)(st.o[rt][db][i] * scaled);
                        v = __builtin_bit_cast(bf16x4, f);
                    }
                    *reinterpret_cast<bf16x4 *>(o + db * 16 + 4 * g4) = v;
                }
                if (g4 == 0) {
                    const float m2 = st.m[rt] == kNegInf ? kNegInf : st.m[rt] * c;
                    if (!last) (whole ? p.ws_row + all + row : p.own_piece + piece)[0] = f32x4{m2, l, unscale, 0.f};
                    else if (p.lse) p.lse[row] = (m2 + __builtin_amdgcn_logf(l)) * kLn2;
                }
            }
            fresh = true;
        }
        if (!nxt.ok) break;
        issue(nxt, ids, true);
        cur = nxt;
        nxt = nn;
        ids = ids_after;
    }
}

}  // namespace
}  // namespace tv
