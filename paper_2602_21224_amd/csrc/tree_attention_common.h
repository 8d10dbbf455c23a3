// What the attention kernels are built from: LDS layout and ring, tile loads,
// the period of one wave over one tile, ancestor sets, work tables.
// (tree_attention.hip explains the design.)
#pragma once

#include "tv_internal.h"

namespace tv {
namespace {

#define LDS_AS __attribute__((address_space(3)))
#define GLOBAL_AS __attribute__((address_space(1)))
#define CONST_AS __attribute__((address_space(4)))

constexpr int KT = kKeyTile;           // 64 keys per tile
constexpr int NS = 4;                  // ring stages (a power of two: stage = tile & (NS - 1))
constexpr int kPageCache = 512;        // page ids cached in LDS per segment window
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kRescaleSlack = 8.f;   // keep a stale running max while new scores stay within 2^8 of it

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <int D>
struct Geo {
    static constexpr int kRowBytes = D * 2;
    static constexpr int kChunks = D / 8;                  // 16-byte chunks per row
    static constexpr int kTileBytes = KT * kRowBytes;      // one of K or V
    static constexpr int kStageBytes = 2 * kTileBytes;
    static constexpr int kBlocksPerTile = kTileBytes / 1024;
    static constexpr int kKeysPerBlock = 1024 / kRowBytes;
};

// Chunk swizzle of a key row: 16-byte chunk c of key k lives at position
// c ^ swz(k % chunks). swz swaps the two low bit-fields of the key so that both
// MFMA operand read patterns are free of LDS bank conflicts: 16 consecutive
// keys at one chunk (K fragments), and 4 consecutive keys x 4 adjacent chunks
// (the transposing V reads). It is a bit permutation, so swz(a ^ b) =
// swz(a) ^ swz(b).
template <int C>
__device__ __forceinline__ constexpr int swz(int k) {
    static_assert(C == 8 || C == 16, "rows of 64 or 128 bf16");
    return C == 16 ? (((k & 3) << 2) | ((k >> 2) & 3)) : (((k & 3) << 1) | ((k >> 2) & 1));
}

// Combine a per-row value held by lanes l and l ^ 32 (the two halves of a
// 32x32 MFMA tile column) without going through LDS.
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Maximum of three values in one instruction (scores are never signalling NaNs).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The same over lanes l, l ^ 16, l ^ 32 and l ^ 48 (the four 16-lane rows of a
// 16x16 MFMA tile's column), by the row-pair swap and then the half-wave swap.
__device__ __forceinline__ float rows_max(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float rows_sum(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// LDS objects are separate so the compiler can see that only `g_ring` is a
// target of the asynchronous tile loads.
__shared__ __attribute__((aligned(1024))) unsigned char g_ring[NS * Geo<128>::kStageBytes];
__shared__ unsigned long long g_anc[kMaxNodes][4];
__shared__ unsigned long long g_anc_alt[kMaxNodes][4];
__shared__ int g_jump[2][kMaxNodes];
__shared__ int g_pages[kPageCache];
__shared__ int g_cum[kMaxBatchAttn + 1];
__shared__ int g_len[kMaxBatchAttn];     // clamped prefix length per sequence
__shared__ unsigned short g_nn[kMaxBatchAttn];   // node count per sequence

__device__ __forceinline__ unsigned lds_addr(const void *p) {
    return (unsigned)(size_t)(const LDS_AS void *)p;
}

__device__ __forceinline__ int clamp_len(int L, const AttnParams &p) {
    const int cap = p.max_pages << p.p_shift;
    return L < 0 ? 0 : (L > cap ? cap : L);
}

// Tree tiles row block rb of a sequence with `rows` query rows must visit.
__device__ __forceinline__ int tree_tiles_of_block(int rb, int rows, const AttnParams &p) {
    const int last_row = min((rb + 1) * p.rows_per_block, rows) - 1;
    const int jmax = last_row / p.G + 1;                  // nodes 0 .. jmax-1 may be ancestors
    return (jmax + KT - 1) / KT;
}

__device__ __forceinline__ int row_blocks_of(int rows, const AttnParams &p) {
    return (rows + p.rows_per_block - 1) / p.rows_per_block;
}

// Virtual tiles of one KV head of a sequence with ntp prefix tiles and `rows`
// query rows: per row block the set-up tiles, the prefix and its tree tiles.
__device__ __forceinline__ int tiles_per_head(int ntp, int rows, const AttnParams &p) {
    int t = 0;
    for (int rb = 0; rb < row_blocks_of(rows, p); ++rb)
        t += p.setup_tiles + ntp + tree_tiles_of_block(rb, rows, p);
    return t;
}

__device__ __forceinline__ int nodes_of(int b, const AttnParams &p) {
    if (!p.num_nodes) return p.N;
    const int n = p.num_nodes[b];
    return n < 0 ? 0 : (n > p.N ? p.N : n);
}

// Work of sequence b in "virtual" tiles: every unit counts setup_tiles in
// front of its real tiles (the cost of starting a piece: its set-up and its
// pipeline fill), so that equal shares of virtual tiles balance the work of
// workgroups that start new units against those that do not.
__device__ __forceinline__ int tiles_of_sequence(int L, int nodes, const AttnParams &p) {
    return p.Hkv * tiles_per_head((L + KT - 1) / KT, nodes * p.G, p);
}

// Explicit LDS wait for reads issued through inline assembly; `tie` makes a
// fragment's later uses depend on the wait (volatile asm keeps its order).
template <int N>
__device__ __forceinline__ void lds_wait() {
    asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N) : "memory");
}
template <typename T>
__device__ __forceinline__ void tie(T &x) {
    asm volatile("" : "+v"(x));
}

__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// s_waitcnt through the builtin, so the compiler's own wait insertion knows
// about it. gfx9 encoding: vmcnt in [3:0] and [15:14], expcnt [6:4], lgkmcnt [11:8].
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit field");
    __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

// Largest finite magnitude of a row of parts (0 if there is none). `each` hands the lane's
// values to a function, `over` takes the maximum over the lanes that hold the row. An
// infinity does not set the scale, which would flush the columns beside it to 0: it stays one
// in fp16 whatever it is multiplied by. NaN passes both maxima by.
template <typename Each, typename Over>
__device__ __forceinline__ float row_top(Each each, Over over) {
    float top = 0.f;
    each([&](float x) { top = fmaxf(top, fabsf(x)); });
    top = over(top);
    if (__any(top == __builtin_huge_valf())) {       // rare: the second look is skipped without
        top = 0.f;
        each([&](float x) {
            const float a = fabsf(x);
            top = fmaxf(top, a < __builtin_huge_valf() ? a : 0.f);
        });
        top = over(top);
    }
    return top;
}

// Scale of a row of parts whose largest finite magnitude is `top`, a power of two that
// brings it just below 2^15 of fp16's 65504, and its inverse.
__device__ __forceinline__ float part_scale(float top, float &unscale) {
    int e = __builtin_amdgcn_frexp_expf(top);        // top = f 2^e, 1/2 <= f < 1; 0 for 0
    e = max(e, -100);
    unscale = __builtin_amdgcn_ldexpf(1.f, e - 15);
    return __builtin_amdgcn_ldexpf(1.f, 15 - e);
}

// Exclusive prefix sum of per-sequence tile counts into g_cum[0..B], the
// clamped prefix lengths into g_len[0..B) and the node counts into g_nn:
// wave 0 reads kv_len (and num_nodes) once per lane and scans with cross-lane
// shifts, one barrier for the whole workgroup.
template <int NT>
__device__ void build_cumulative(const AttnParams &p) {
    if (threadIdx.x < kWave) {
        const int lane = threadIdx.x;
        int carry = 0;
        for (int b0 = 0; b0 < p.B; b0 += kWave) {
            const int b = b0 + lane;
            const int L = b < p.B ? clamp_len(p.kv_len[b], p) : 0;
            const int nb = b < p.B ? nodes_of(b, p) : 0;
            const int t = b < p.B ? tiles_of_sequence(L, nb, p) : 0;
            int x = t;                                   // inclusive scan over the wave
            #pragma unroll
            for (int off = 1; off < kWave; off <<= 1) {
                const int y = __shfl_up(x, off);
                if (lane >= off) x += y;
            }
            if (b < p.B) {
                g_cum[b] = carry + x - t;
                g_len[b] = L;
                g_nn[b] = (unsigned short)nb;
            }
            carry += __shfl(x, kWave - 1);
        }
        if (lane == 0) g_cum[p.B] = carry;
    }
    __syncthreads();
}

// Piece set-up for pages shorter than a load block: page ids of pages
// [first, first + kPageCache) of sequence b (as far as it has them) into
// g_pages; all loads are issued before any is waited for.
template <int NT>
__device__ void load_pages(const AttnParams &p, int b, int first, int npages) {
    constexpr int PPT = (kPageCache + NT - 1) / NT;
    const int tid = threadIdx.x;
    const int n = min(kPageCache, npages - first);
    int pg[PPT];
    #pragma unroll
    for (int k = 0; k < PPT; ++k) {
        const int i = tid + k * NT;
        pg[k] = i < n ? p.page_table[(size_t)b * p.max_pages + first + i] : -1;
    }
    #pragma unroll
    for (int k = 0; k < PPT; ++k) {
        const int i = tid + k * NT;
        if (i < n) g_pages[i] = (pg[k] >= 0 && pg[k] < p.num_pages) ? pg[k] : -1;
    }
    __syncthreads();
}

// Ancestor sets of a tree of at most 64 nodes, by one wave and without
// barriers: lane i holds node i's set (one 64-bit word, reflexive) and the
// ancestor 2^k steps up; each round ORs in that ancestor's set and jumps
// twice as far (cross-lane reads see the values of the previous round), until
// no lane has an ancestor left. The caller's next workgroup barrier publishes
// g_anc.
// `pi` is node `lane`'s parent as loaded by the caller (any value for lanes >= N).
__device__ void build_ancestor_masks_wave(const AttnParams &p, int pi) {
    const int lane = threadIdx.x & (kWave - 1);
    int j = -1;
    if (lane < p.N) j = (pi < -1 || pi >= lane) ? -1 : pi;   // contract violation: treat as a root
    unsigned long long anc = lane < p.N ? (1ull << lane) : 0ull;
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
    if (lane < p.N) {
        g_anc[lane][0] = anc;
        g_anc[lane][1] = 0ull;
        g_anc[lane][2] = 0ull;
        g_anc[lane][3] = 0ull;
    }
}

// The same for up to kMaxNodes nodes, still one wave and no workgroup
// barrier: lane l owns nodes l, l + 64, ...; sets and jumps of the previous
// round are read from LDS (double buffered), and a wave-local wait for the
// LDS writes separates the rounds.
__device__ void build_ancestor_masks_wave_lds(const AttnParams &p, int b) {
    constexpr int K = kMaxNodes / kWave;
    const int lane = threadIdx.x & (kWave - 1);
    int jmp[K];
    #pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = lane + k * kWave;
        jmp[k] = -1;
        if (i < p.N) {
            const int pi = p.parent[(size_t)b * p.N + i];
            jmp[k] = (pi < -1 || pi >= i) ? -1 : pi;
            #pragma unroll
            for (int w = 0; w < 4; ++w) g_anc[i][w] = (w == (i >> 6)) ? (1ull << (i & 63)) : 0ull;
            g_jump[0][i] = jmp[k];
        }
    }
    int cur = 0;
    for (;;) {
        bool more = false;
        #pragma unroll
        for (int k = 0; k < K; ++k) more |= jmp[k] >= 0;
        if (!__any(more)) break;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        unsigned long long(*src)[4] = cur == 0 ? g_anc : g_anc_alt;
        unsigned long long(*dst)[4] = cur == 0 ? g_anc_alt : g_anc;
        #pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = lane + k * kWave;
            if (i >= p.N) continue;
            const int j = jmp[k];
            if (j >= 0) {
                #pragma unroll
                for (int w = 0; w < 4; ++w) dst[i][w] = src[i][w] | src[j][w];
                jmp[k] = g_jump[cur][j];
            } else {
                #pragma unroll
                for (int w = 0; w < 4; ++w) dst[i][w] = src[i][w];
            }
            g_jump[cur ^ 1][i] = jmp[k];
        }
        cur ^= 1;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (cur == 1) {
        #pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = lane + k * kWave;
            if (i < p.N)
                #pragma unroll
                for (int w = 0; w < 4; ++w) g_anc[i][w] = g_anc_alt[i][w];
        }
    }
}

template <int D, int NW, bool SMALL>
struct TileIssue {
    using Gm = Geo<D>;
    static constexpr int kLoadsPerWave = Gm::kBlocksPerTile / NW;   // per K (or V) tile
    static constexpr int LPT = kLoadsPerWave;
    static constexpr int KPB = Gm::kKeysPerBlock;     // keys per 1 KB load block
    static constexpr int C = Gm::kChunks;
    static_assert(LPT * NW == Gm::kBlocksPerTile, "blocks split evenly over waves");

    // Wave-uniform addresses of this wave's load blocks of one tile: the K and
    // V row of the block's first key, and how many of its KPB keys exist.
    struct Blocks {
        const char *k[LPT];
        const char *v[LPT];
        int nv[LPT];
    };

    int kib;                                          // this lane's key within a block
    unsigned row_off;                                 // kib * key row stride (bytes)
    unsigned chunk_off[LPT];                          // swizzled chunk offset per load
    unsigned lane_off[LPT];                           // i * KPB rows + row_off + chunk_off[i]
    // per unit
    const char *kc_g, *vc_g;                          // cache base + KV head g
    const char *kt_g, *vt_g;                          // tree row of node 0, KV head g
    unsigned row_bytes, page_bytes;                   // key row of all KV heads; one page
    int L, ntp, nodes;

    __device__ __forceinline__ void init(int wave_u, int lane, const AttnParams &p) {
        row_bytes = (unsigned)(p.Hkv * D * 2);
        page_bytes = row_bytes << p.p_shift;
        kib = lane / C;
        row_off = kib * row_bytes;
        #pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int kb = wave_u * LPT + i;
            chunk_off[i] = (unsigned)(((lane % C) ^ swz<C>((kb * KPB + kib) % C)) * 16);
            lane_off[i] = (unsigned)(i * KPB) * row_bytes + row_off + chunk_off[i];
        }
    }

    // Common case of a prefix tile: every row of the tile exists, this wave's
    // LPT blocks (consecutive keys) lie in one page, and that page id (pg0,
    // the page of the wave's first key) is valid. Then block i starts
    // i * KPB rows after `off`, the byte offset of the wave's first key row
    // from the cache base of KV head g. Returns false otherwise.
    __device__ __forceinline__ bool fast_offset(const AttnParams &p, int t, int wave_u, int pg0,
                                                unsigned long long &off) const {
        const int pos_w = t * KT + wave_u * LPT * KPB;
        if (LPT * KPB > p.P || t >= ntp || t * KT + KT > L || (unsigned)pg0 >= (unsigned)p.num_pages)
            return false;
        off = (unsigned long long)(unsigned)pg0 * page_bytes + (unsigned)(pos_w & (p.P - 1)) * row_bytes;
        return true;
    }

    // Direct-to-LDS loads of this wave's blocks of one K (or V) tile of the
    // common case (see fast_offset) into ring stage `stage`.
    __device__ __forceinline__ void issue_fast(unsigned long long off, bool is_v, int stage,
                                               int wave_u) const {
        unsigned char *dst = g_ring + stage * Gm::kStageBytes + (is_v ? Gm::kTileBytes : 0);
        const char *base = (is_v ? vc_g : kc_g) + off;
        #pragma unroll
        for (int i = 0; i < LPT; ++i)
            __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)(base + lane_off[i]),
                                             (LDS_AS void *)(dst + (wave_u * LPT + i) * 1024), 16, 0, 0);
    }

    __device__ __forceinline__ void set_unit(const AttnParams &p, int b, int g, int L_, int ntp_,
                                             int nodes_) {
        L = L_;
        ntp = ntp_;
        nodes = nodes_;
        kc_g = reinterpret_cast<const char *>(p.k_cache + (size_t)g * D);
        vc_g = reinterpret_cast<const char *>(p.v_cache + (size_t)g * D);
        kt_g = reinterpret_cast<const char *>(p.k_tree + ((size_t)b * p.N * p.Hkv + g) * D);
        vt_g = reinterpret_cast<const char *>(p.v_tree + ((size_t)b * p.N * p.Hkv + g) * D);
    }

    // Page ids of this wave's load blocks of prefix tile t, by scalar loads
    // through the constant address space: the ids land in SGPRs without
    // touching LDS. The index is clamped into the table row, so the load is
    // always in bounds; blocks() decides whether an id is used. Callers fetch
    // one tile period before the loads are issued, and nothing here waits for
    // the result.
    __device__ __forceinline__ void fetch_pages(const AttnParams &p, int b, int t, int wave_u,
                                                int (&pg)[LPT]) const {
        const CONST_AS int32_t *row =
            (const CONST_AS int32_t *)(p.page_table + (size_t)b * p.max_pages);
        #pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int pos0 = t * KT + (wave_u * LPT + i) * KPB;
            pg[i] = SMALL ? -1 : row[min(max(pos0 >> p.p_shift, 0), p.max_pages - 1)];
        }
    }

    // Block addresses of tile t. A block with no existing row (past the prefix,
    // past the sequence's nodes, or with an invalid page id) points at tree
    // node 0's row, which is always readable and finite; its rows are masked
    // later.
    __device__ __forceinline__ Blocks blocks(const AttnParams &p, int t, int wave_u,
                                             const int (&pg)[LPT]) const {
        Blocks r;
        if (t < ntp) {
            const bool full = t * KT + KT <= L;            // every row of the tile exists
            const int pos_w = t * KT + wave_u * LPT * KPB;  // first key of this wave's blocks
            #pragma unroll
            for (int i = 0; i < LPT; ++i) {
                const int pos0 = pos_w + i * KPB;
                const bool ok = (unsigned)pg[i] < (unsigned)p.num_pages && (full || pos0 < L);
                const size_t off = (size_t)(unsigned)pg[i] * page_bytes +
                                   (unsigned)((pos0 & (p.P - 1)) * row_bytes);
                r.k[i] = ok ? kc_g + off : kt_g;
                r.v[i] = ok ? vc_g + off : vt_g;
                r.nv[i] = !ok ? 0 : (full ? KPB : min(L - pos0, KPB));
            }
        } else {
            #pragma unroll
            for (int i = 0; i < LPT; ++i) {
                const int j0 = (t - ntp) * KT + (wave_u * LPT + i) * KPB;
                const int nv = min(max(nodes - j0, 0), KPB);
                const unsigned off = nv > 0 ? (unsigned)j0 * (unsigned)row_bytes : 0u;
                r.k[i] = kt_g + off;
                r.v[i] = vt_g + off;
                r.nv[i] = nv;
            }
        }
        return r;
    }

    // Direct-to-LDS loads of this wave's blocks of one K (or V) tile into ring
    // stage `stage`. A key of a block behind its last existing one reads the block's
    // first row of K, whose scores are replaced. Its weight in V is 0, and 0 times an
    // infinity of a cached row is NaN, so there it reads tree node 0's row, in a load of
    // its own: a selected address cost the eight-wave kernels spills, and a load more than
    // the waits count makes them wait for more, never for less. (With pages shorter than
    // a block only tree tiles come here.)
    __device__ __forceinline__ void issue(const Blocks &bl, bool is_v, int stage, int wave_u) const {
        unsigned char *dst = g_ring + stage * Gm::kStageBytes + (is_v ? Gm::kTileBytes : 0);
        #pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const bool in = kib < bl.nv[i];
            const char *addr = (is_v ? bl.v[i] : bl.k[i]) + ((in ? row_off : 0u) + chunk_off[i]);
            LDS_AS void *to = (LDS_AS void *)(dst + (wave_u * LPT + i) * 1024);
            if (SMALL || !is_v || in)
                __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)addr, to, 16, 0, 0);
            else
                __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)(vt_g + chunk_off[i]), to, 16, 0, 0);
        }
    }

    // Pages shorter than a load block: every lane looks up its own page in the
    // LDS page-id window (prefix tiles only).
    __device__ __forceinline__ void issue_small(const AttnParams &p, int t, bool is_v, int page_first,
                                                int wave_u) const {
        unsigned char *dst = g_ring + (t & (NS - 1)) * Gm::kStageBytes + (is_v ? Gm::kTileBytes : 0);
        #pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int pos = t * KT + (wave_u * LPT + i) * KPB + kib;
            const char *row = is_v ? vt_g : kt_g;
            if (pos < L) {
                const int id = g_pages[(pos >> p.p_shift) - page_first];
                if (id >= 0)
                    row = (is_v ? vc_g : kc_g) + (size_t)(unsigned)id * page_bytes + (size_t)(pos & (p.P - 1)) * row_bytes;
            }
            __builtin_amdgcn_global_load_lds((const GLOBAL_AS void *)(row + chunk_off[i]),
                                             (LDS_AS void *)(dst + (wave_u * LPT + i) * 1024), 16, 0, 0);
        }
    }
};

// Wait until at most n of this wave's vector-memory operations are still in
// flight; a count without its own case waits for the next smaller one.
__device__ __forceinline__ void wait_vm_at_most(int n) {
    if (n >= 63) wait_vmcnt<63>();
    else if (n >= 48) wait_vmcnt<48>();
    else if (n >= 32) wait_vmcnt<32>();
    else if (n >= 24) wait_vmcnt<24>();
    else if (n >= 16) wait_vmcnt<16>();
    else if (n >= 12) wait_vmcnt<12>();
    else if (n >= 8) wait_vmcnt<8>();
    else if (n >= 6) wait_vmcnt<6>();
    else if (n >= 4) wait_vmcnt<4>();
    else if (n >= 2) wait_vmcnt<2>();
    else if (n >= 1) wait_vmcnt<1>();
    else wait_vmcnt<0>();
}

// LDS-read wait with a count that is a constant once the caller is unrolled.
__device__ __forceinline__ void lds_wait_n(int n) {
    switch (n) {
        case 0: lds_wait<0>(); break;
        case 1: lds_wait<1>(); break;
        case 2: lds_wait<2>(); break;
        case 3: lds_wait<3>(); break;
        case 4: lds_wait<4>(); break;
        case 5: lds_wait<5>(); break;
        case 6: lds_wait<6>(); break;
        case 7: lds_wait<7>(); break;
        case 8: lds_wait<8>(); break;
        default: lds_wait<0>(); break;
    }
}

// Per-wave state of one piece: Q fragments (MFMA B operand), O^T
// accumulators, the probabilities of the tile whose PV product is pending,
// running max and sum.
template <int D>
struct WaveState {
    static constexpr int NKS = D / 16;     // MFMA k-steps over the head dim
    static constexpr int NDT = D / 32;     // 32-wide head-dim tiles of the output
    bf16x8 qf[NKS];
    f32x16 o[NDT];
    u32x4 pb[4];                           // P^T as bf16 pairs, 16 keys per k-step
    float m_run;                           // running max (raw score units)
    float msc;                             // m_run * scale_log2 (0 while m_run is -inf)
    float l_run;                           // this lane's part of the running sum
};

// Visible keys of tile j for the lane's row: every key of a full prefix tile
// (masked = false, wave-uniform), the keys below the prefix length on the last
// prefix tile, the node's ancestors on a tree tile. Bit k of (vis_hi:vis_lo)
// is the key the lane holds at position k of a half-0 lane (the lane's own
// half already shifted in).
struct TileMask {
    bool masked;
    unsigned vis_lo, vis_hi;
};

// Key position (within the tile) of accumulator element r of half hf, for a
// lane of half 0; a lane of half 1 holds the key 4 positions later.
__host__ __device__ constexpr int key_of(int hf, int r) { return hf * 32 + (r >> 2) * 8 + (r & 3); }

// Exponentials of 2 scores of one tile into a bf16 pair of P^T and the
// running sum: x = 2^(s * c - msc).
// The results are tied (empty volatile asm) so that the computation stays in
// the MFMA slot it was written in instead of sinking to its first use.
__device__ __forceinline__ unsigned exp_pair(float s0, float s1, float c, float msc, float &sum) {
    const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s0, c, -msc));
    const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1, c, -msc));
    sum += x0 + x1;
    const bf16x2 pr = {(__bf16)x0, (__bf16)x1};
    unsigned u = __builtin_bit_cast(unsigned, pr);
    tie(u);
    tie(sum);
    return u;
}

// One tile period of one wave.
//   CUR:  part A computes tile j's scores S^T = K_j Q^T into s0 (keys 0..31)
//         and s1 (keys 32..63); part B masks them, takes their maximum,
//         decides the running maximum and exponentiates half 0 into P^T.
//   PREV: the first half of part A exponentiates the previous tile's half 1
//         (in s1, consumed before this tile's half-1 products overwrite it);
//         part B adds P^T V_{j-1} to O.
// The VALU slices sit between the MFMAs of their part, so the matrix pipe and
// the VALU of one wave overlap; two 16-register score halves are alive at any
// time. LDS operand reads run two MFMAs ahead with explicit waits.
template <int D, bool PREV, bool CUR>
__device__ __forceinline__ void tile_period(WaveState<D> &st, f32x16 &sc0, f32x16 &sc1,
                                            unsigned kaddr, unsigned vaddr, const TileMask &mk,
                                            float c) {
    f32x16 *sc[2] = {&sc0, &sc1};
    using Gm = Geo<D>;
    constexpr int NKS = D / 16, NDT = D / 32;
    constexpr int C = Gm::kChunks;
    constexpr int SA = 2 * NKS;            // part A slots: one S MFMA each
    constexpr int SB = 4 * NDT;            // part B slots: one PV MFMA each
    constexpr int NSLOT = SA + SB;
    constexpr int R = 2;                   // operand reads run this many slots ahead
    constexpr int PPA = 8 / NKS;                       // half-1 pairs per slot of part A's first half
    // first part-B slot of the half-0 pairs: after the decision (slot 5) and
    // after the PV MFMAs that read P^T k-steps 0 and 1 have issued
    constexpr int B0 = 2 * NDT > 6 ? 2 * NDT : 6;
    constexpr int PPB = (8 + (SB - B0) - 1) / (SB - B0);   // half-0 pairs per part-B slot
    static_assert(NKS <= 8 && 8 % NKS == 0 && SB > B0, "slice shapes");
    auto active = [](int s) { return s < SA ? CUR : PREV; };
    auto ops = [&](int s) { return (s < NSLOT && active(s)) ? (s < SA ? 1 : 2) : 0; };
    u32x4 kb[SA];
    u32x2 vb[SB][2];
    auto issue_reads = [&](int s) {
        if (s >= NSLOT || !active(s)) return;
        if (s < SA) {
            const int hf = s / NKS, ks = s % NKS;
            asm volatile("ds_read_b128 %0, %1 offset:%2"
                         : "=v"(kb[s])
                         : "v"(kaddr ^ ((unsigned)ks << 5)), "i"(hf * 32 * Gm::kRowBytes));
        } else {
            const int b = s - SA, kk = b / NDT, dt = b % NDT;
            #pragma unroll
            for (int rr = 0; rr < 2; ++rr) {
                const unsigned flip = (unsigned)((dt * 4) ^ swz<C>((rr * 8) % C)) << 4;
                asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2"
                             : "=v"(vb[b][rr])
                             : "v"(vaddr ^ flip), "i"((kk * 16 + rr * 8) * Gm::kRowBytes));
            }
        }
    };
    float psa = 0.f, psb = 0.f;
    float m8[4];
    float alpha = 1.f;
    bool any_raise = false;
    #pragma unroll
    for (int s = 0; s < R; ++s) issue_reads(s);
    #pragma unroll
    for (int s = 0; s < NSLOT; ++s) {
        issue_reads(s + R);
        if (active(s)) {
            int newer = 0;
            #pragma unroll
            for (int k = 1; k <= R; ++k) newer += ops(s + k);
            lds_wait_n(newer);
            if (s < SA) {
                const int hf = s / NKS, ks = s % NKS;
                tie(kb[s]);
                const f32x16 acc = ks == 0 ? f32x16{} : *sc[hf];   // a chain starts from zero
                *sc[hf] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kb[s]),
                                                                  st.qf[ks], acc, 0, 0, 0);
            } else {
                const int b = s - SA, kk = b / NDT, dt = b % NDT;
                tie(vb[b][0]);
                tie(vb[b][1]);
                const u32x4 a = {vb[b][0][0], vb[b][0][1], vb[b][1][0], vb[b][1][1]};
                st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, st.pb[kk]), st.o[dt],
                    0, 0, 0);
            }
        }
        if (PREV && s < NKS) {
            // pairs of the previous tile's half 1 (keys 32 + 2i, 33 + 2i: P^T
            // k-steps 2, 3), all before slot NKS overwrites s1
            #pragma unroll
            for (int u = 0; u < PPA; ++u) {
                const int i = s * PPA + u, kk = 2 + (i >> 2), w = i & 3;
                st.pb[kk][w] = exp_pair(sc1[2 * i], sc1[2 * i + 1], c, st.msc, psa);
            }
        }
        if (PREV && s == NKS - 1) st.l_run += psa;
        if (CUR && s == SA + 1 && mk.masked) {
            // the last prefix tile or a tree tile: invisible keys become -inf
            // (selected, never added), in place
            #pragma unroll
            for (int hf = 0; hf < 2; ++hf)
                #pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = key_of(hf, r);
                    const unsigned word = k < 32 ? mk.vis_lo : mk.vis_hi;
                    (*sc[hf])[r] = ((word >> (k & 31)) & 1u) ? (*sc[hf])[r] : kNegInf;
                }
        }
        if (CUR && s >= SA + 1 && s < SA + 5) {
            // maximum of 8 of this tile's scores (chunk q: half q / 2, elements
            // 8 (q % 2) .. +8)
            const int q = s - SA - 1, hf = q >> 1, r0 = (q & 1) * 8;
            const f32x16 &v = *sc[hf];
            const float a = max3(v[r0], v[r0 + 1], v[r0 + 2]);
            const float b = max3(v[r0 + 3], v[r0 + 4], v[r0 + 5]);
            m8[q] = max3(a, b, max3(v[r0 + 6], v[r0 + 7], v[r0 + 7]));
            tie(m8[q]);
        }
        if (CUR && s == SA + 5) {
            // The running max is only raised when a score exceeds it by more
            // than kRescaleSlack (log2 units), so O is rarely rescaled. The
            // sum is rescaled here; O after this period's PV products.
            const float tmax = halves_max(max3(m8[0], m8[1], max3(m8[2], m8[3], m8[3])));
            const bool raise = tmax * c > st.m_run * c + kRescaleSlack;
            any_raise = __any(raise);
            if (any_raise) {
                const float m_new = raise ? tmax : st.m_run;
                alpha = (st.m_run == kNegInf) ? 0.f
                        : __builtin_amdgcn_exp2f((st.m_run - m_new) * c);
                st.l_run *= alpha;
                st.m_run = m_new;
            }
            st.msc = (st.m_run == kNegInf) ? 0.f : st.m_run * c;
        }
        if (CUR && s >= SA + B0) {
            #pragma unroll
            for (int u = 0; u < PPB; ++u) {
                const int i = (s - SA - B0) * PPB + u;     // pair i of half 0: keys 2i, 2i + 1
                if (i < 8) st.pb[i >> 2][i & 3] = exp_pair(sc0[2 * i], sc0[2 * i + 1], c, st.msc, psb);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if (CUR) {
        st.l_run += psb;
        if (any_raise) {
            #pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
                #pragma unroll
                for (int r = 0; r < 16; ++r) st.o[dt][r] *= alpha;
        }
    }
}

// ---- units of at most 16 query rows (the paper's own MHA shape: 12 nodes x 1
// head per KV head). Every row tile of the main scheme would be mostly empty,
// so here the workgroup's waves take the unit's tiles in turn (tile j belongs
// to wave j mod NW) and compute it whole with v_mfma_f32_16x16x32_bf16: keys on
// M (16 per block, 4 blocks per tile), the 16 rows on N, head dim on K. Lane l
// holds row l % 16; in a 16x16 accumulator it holds entries m = 4 (l / 16) + i,
// i < 4, so S gives it keys 16 kb + 4 (l / 16) + i of every key block kb. The
// PV product takes P^T straight from there: its k-step over key blocks (kb0,
// kb1) pairs k = 8 (l / 16) + i with key 16 kb0 + 4 (l / 16) + i and
// k = 8 (l / 16) + 4 + i with key 16 kb1 + 4 (l / 16) + i, and the V^T operand
// is read with the same key order through ds_read_b64_tr_b16 (a 16-lane group
// reads 4 key rows x 16 head-dim columns; lane i of the group receives column
// i of the 4 rows). Each wave keeps its own running max, sum and O^T for its
// tiles; the waves' states are combined with the log-sum-exp rule at the end
// of the piece. Tile loads stay cooperative (all waves, one barrier per tile),
// and with one wave computing per tile the period is bound by the loads.
template <int D>
struct NarrowState {
    static constexpr int NKS = D / 32;     // k-steps over the head dim (S)
    static constexpr int NDB = D / 16;     // 16-wide head-dim blocks of O^T
    bf16x8 qf[NKS];
    f32x4 o[NDB];
    float m_run, msc, l_run;
};

// Tile j for the owning wave. kaddr/vaddr: the stage's K and V tile bases (LDS
// byte addresses); vis: the visible keys of the lane's row (bit = key in tile),
// all ones for a full prefix tile.
template <int D>
__device__ __forceinline__ void narrow_tile(NarrowState<D> &st, unsigned kbase, unsigned vbase,
                                            bool masked, unsigned long long vis, float c, int lane) {
    using Gm = Geo<D>;
    constexpr int C = Gm::kChunks;
    constexpr int NKS = D / 32, NDB = D / 16;
    const int g = lane >> 4, i16 = lane & 15;
    // S^T blocks; the K reads of block kb + 1 are in flight during block kb's MFMAs
    f32x4 sb[4];
    u32x4 a[2][NKS];
    auto read_k = [&](int kb, u32x4 (&dst)[NKS]) {
        const int key = kb * 16 + i16;
        const unsigned row = kbase + key * Gm::kRowBytes;
        #pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
            asm volatile("ds_read_b128 %0, %1" : "=v"(dst[ks])
                         : "v"(row + ((unsigned)((4 * ks + g) ^ swz<C>(key % C)) << 4)));
    };
    read_k(0, a[0]);
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
        if (kb + 1 < 4) {
            read_k(kb + 1, a[(kb + 1) & 1]);
            lds_wait<NKS>();
        } else {
            lds_wait<0>();
        }
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        #pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            tie(a[kb & 1][ks]);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[kb & 1][ks]),
                                                          st.qf[ks], acc, 0, 0, 0);
        }
        sb[kb] = acc;
    }
    if (masked) {
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb)
            #pragma unroll
            for (int i = 0; i < 4; ++i)
                sb[kb][i] = ((vis >> (kb * 16 + 4 * g + i)) & 1ull) ? sb[kb][i] : kNegInf;
    }
    float mt = kNegInf;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb) mt = fmaxf(mt, fmaxf(fmaxf(sb[kb][0], sb[kb][1]), fmaxf(sb[kb][2], sb[kb][3])));
    mt = rows_max(mt);
    const bool raise = mt * c > st.m_run * c + kRescaleSlack;
    if (__any(raise)) {
        const float m_new = raise ? mt : st.m_run;
        const float alpha = (st.m_run == kNegInf) ? 0.f : __builtin_amdgcn_exp2f((st.m_run - m_new) * c);
        st.l_run *= alpha;
        #pragma unroll
        for (int db = 0; db < NDB; ++db)
            #pragma unroll
            for (int i = 0; i < 4; ++i) st.o[db][i] *= alpha;
        st.m_run = m_new;
    }
    st.msc = (st.m_run == kNegInf) ? 0.f : st.m_run * c;
    bf16x8 pb[2];
    float ps = 0.f;
    #pragma unroll
    for (int kb = 0; kb < 4; ++kb)
        #pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sb[kb][i], c, -st.msc));
            ps += x;
            pb[kb >> 1][(kb & 1) * 4 + i] = (__bf16)x;
        }
    st.l_run += ps;
    // O^T += V^T P^T, two k-steps of 32 keys; step q = kst * NDB + db, its two
    // transposing reads issued two steps ahead
    constexpr int NQ = 2 * NDB;
    u32x2 v[NQ][2];
    auto read_v = [&](int q) {
        const int kst = q / NDB, db = q % NDB;
        #pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int key = (2 * kst + r) * 16 + 4 * g + (i16 >> 2);
            const int chunk = 2 * db + ((i16 & 3) >> 1);
            const unsigned addr = vbase + key * Gm::kRowBytes +
                                  ((unsigned)(chunk ^ swz<C>(key % C)) << 4) + (i16 & 1) * 8;
            asm volatile("ds_read_b64_tr_b16 %0, %1" : "=v"(v[q][r]) : "v"(addr));
        }
    };
    read_v(0);
    read_v(1);
    #pragma unroll
    for (int q = 0; q < NQ; ++q) {
        if (q + 2 < NQ) {
            read_v(q + 2);
            lds_wait<4>();
        } else if (q + 1 < NQ) {
            lds_wait<2>();
        } else {
            lds_wait<0>();
        }
        tie(v[q][0]);
        tie(v[q][1]);
        const int kst = q / NDB, db = q % NDB;
        const u32x4 av = {v[q][0][0], v[q][0][1], v[q][1][0], v[q][1][1]};
        st.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, av), pb[kst],
                                                           st.o[db], 0, 0, 0);
    }
}

}  // namespace
}  // namespace tv
