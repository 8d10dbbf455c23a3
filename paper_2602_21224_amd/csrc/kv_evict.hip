// Eviction from the paged cache by accumulated attention weight, for gfx950.
//
// The slots of a (sequence, KV head) fall into three kinds that rank before
// one another (fixed, recent, others); the budget cuts one of the last two,
// and there the cut is the k-th largest weight. One workgroup per (sequence,
// KV head) finds it:
//   * Every wave owns one run of slots and holds their weights in registers
//     (four neighbouring slots per lane and load), so the passes below read
//     nothing again; caches of more than kSlots<ITER> slots per head re-read
//     theirs (L2) in the same passes.
//   * Radix select over the order-preserving 32-bit keys in digits of 11, 11 and
//     10 bits: three histograms in LDS. Where a wave's keys all have one digit
//     (weights of zero) it adds their number once, so equal weights cost no
//     serialised additions. The bin that holds the cut is found by a suffix sum
//     over all threads.
//   * Among the keys equal to the cut the lowest slots stay. Every wave counts
//     its own run, one exchange of the waves' counts gives each its offset, and
//     so the evicted slots below the kept length and the kept slots past it are
//     listed in slot order with three barriers, whatever the length.
// The k-th slot of the first list takes the row of the k-th of the second:
// sources lie past the kept length and destinations below it, so no move reads
// what another wrote, and only rows that have to move do. A second kernel moves
// them with the whole chip; where there can be few, the first does.
#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kBins = 2048;
constexpr int kMoveThreads = 256;
constexpr int kFewMoves = 128;      // rows that the selecting workgroup moves itself

// Slots in registers: ITER loads of 4 per lane.
template <int NT, int ITER>
constexpr int kSlots = NT * 4 * ITER;

__device__ __forceinline__ int wave_sum(int x) {
    #pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
__device__ __forceinline__ int wave_prefix(int x) {          // inclusive
    const int lane = threadIdx.x & (kWave - 1);
    #pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    return x;
}

// Moves of one (sequence, KV head): threads tid, tid + step, ... of all that share
// them take 16-byte pieces of the rows' K and V.
__device__ __forceinline__ void move_rows(const EvictParams &p, int b, int g, int n, int tid, int step) {
    const int T = p.max_pages << p.p_shift;
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    const int32_t *holes = p.moves + base, *from = holes + T / 2;
    const int32_t *table = p.page_table + (size_t)b * p.max_pages;
    const int chunks = p.D / 8, mask = (1 << p.p_shift) - 1;
    for (int i = tid; i < n * chunks; i += step) {
        const int m = i / chunks, c = i - m * chunks;
        const int dst = holes[m], src = from[m];
        if (c == 0) {
            p.weight_out[base + dst] = p.weight[base + src];
            p.position_out[base + dst] = p.position[base + src];
        }
        const int pd = table[dst >> p.p_shift], ps = table[src >> p.p_shift];
        if (pd < 0 || pd >= p.num_pages || ps < 0 || ps >= p.num_pages) continue;
        const size_t d = ((((size_t)pd << p.p_shift) + (dst & mask)) * p.Hkv + g) * p.D + c * 8;
        const size_t s = ((((size_t)ps << p.p_shift) + (src & mask)) * p.Hkv + g) * p.D + c * 8;
        const u16x8 k = *reinterpret_cast<const u16x8 *>(p.k_cache + s);
        const u16x8 v = *reinterpret_cast<const u16x8 *>(p.v_cache + s);
        *reinterpret_cast<u16x8 *>(p.k_cache + d) = k;
        *reinterpret_cast<u16x8 *>(p.v_cache + d) = v;
    }
}

template <int NT, int ITER>
__global__ __launch_bounds__(NT) void evict_select_kernel(EvictParams p) {
    constexpr int NW = NT / kWave;
    __shared__ int hist[3][kBins];
    __shared__ int part[4][NW];
    __shared__ int s_bin[3][2];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int lane = tid & (kWave - 1), wave = tid / kWave;
    const int T = p.max_pages << p.p_shift;
    const int L = min(max(p.kv_len[b], 0), T);
    const int fixed = p.fixed_len ? min(max(p.fixed_len[b], 0), L) : 0;
    const int keep = min(L, max(p.budget, fixed));
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    const float *weight = p.weight + base;
    const int32_t *position = p.position + base;
    float *wout = p.weight_out != p.weight ? p.weight_out + base : nullptr;
    int32_t *pout = p.position_out != p.position ? p.position_out + base : nullptr;
    const long long newest = (long long)p.seen[b] - p.recent;
    if (g == 0 && tid == 0) p.kept_len[b] = keep;
    int *count = p.count + (size_t)b * p.Hkv + g;
    // this wave's run of slots: `iters` loads of 256
    const int iters = (L + NT * 4 - 1) / (NT * 4);
    const int first = wave * iters * 4 * kWave + lane * 4;
    const bool held = iters <= ITER;
    const bool wide = p.vector_slots;

    float w[ITER][4];
    unsigned int recent[(ITER + 7) / 8] = {};         // bit 4 i + e: slot e of load i is a recent one
    auto load = [&](int t, float (&x)[4], int (&y)[4]) {
        if (wide && t + 4 <= L) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(weight + t);
            const i32x4 c = *reinterpret_cast<const i32x4 *>(position + t);
            #pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = a[e]; y[e] = c[e]; }
        } else {
            #pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = t + e < L ? weight[t + e] : 0.f;
                y[e] = t + e < L ? position[t + e] : 0;
            }
        }
    };
    // `body(t, x, r)` over this lane's slots: t the first of four, x their weights, bit e
    // of r whether slot t + e is recent
    auto each = [&](auto body) {
        if (held) {
            #pragma unroll
            for (int i = 0; i < ITER; ++i)
                if (i < iters) body(first + i * 4 * kWave, w[i], recent[i / 8] >> (i % 8 * 4));
        } else {
            for (int i = 0; i < iters; ++i) {
                const int t = first + i * 4 * kWave;
                float x[4];
                int y[4];
                load(t, x, y);
                unsigned int r = 0u;
                #pragma unroll
                for (int e = 0; e < 4; ++e) r |= (y[e] >= newest ? 1u : 0u) << e;
                body(t, x, r);
            }
        }
    };

    for (int i = tid; i < 3 * kBins; i += NT) hist[i / kBins][i % kBins] = 0;
    // weights and positions, once; arrays of their own take what may stay where it is
    // (slots that are evicted are written again by their moves)
    int recents = 0;
    auto first_look = [&](int t, const float (&x)[4], const int (&y)[4]) {
        unsigned int r = 0u;
        #pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (t + e >= fixed && t + e < L && y[e] >= newest) { r |= 1u << e; ++recents; }
            if (t + e < keep) {
                if (wout) wout[t + e] = x[e];
                if (pout) pout[t + e] = y[e];
            }
        }
        return r;
    };
    if (held) {
        int y[ITER][4];
        #pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (i < iters) load(first + i * 4 * kWave, w[i], y[i]);
        #pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (i < iters) recent[i / 8] |= first_look(first + i * 4 * kWave, w[i], y[i]) << (i % 8 * 4);
    } else {
        for (int i = 0; i < iters; ++i) {
            float x[4];
            int y[4];
            load(first + i * 4 * kWave, x, y);
            first_look(first + i * 4 * kWave, x, y);
        }
    }
    if (keep == L) {
        if (tid == 0) *count = 0;
        return;
    }
    recents = wave_sum(recents);
    if (lane == 0) part[0][wave] = recents;
    __syncthreads();
    recents = 0;
    #pragma unroll
    for (int v = 0; v < NW; ++v) recents += part[0][v];

    // which kind the budget cuts, and how many of it stay
    const bool cut_recent = recents >= keep - fixed;
    const int want = cut_recent ? keep - fixed : keep - fixed - recents;
    const unsigned int flip = cut_recent ? 0u : 15u;
    unsigned int cut = 0u;
    int left = want;                     // of those equal to the cut, how many stay
    if (want > 0) {
        #pragma unroll
        for (int d = 0; d < 3; ++d) {
            const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bins = d == 2 ? 1024 : 2048;
            each([&](int t, const float (&x)[4], unsigned int r) {
                r ^= flip;               // slots of the cut kind
                #pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const unsigned int k = order_key(x[e]);
                    const bool in = t + e >= fixed && t + e < L && ((r >> e) & 1u) &&
                                    (d == 0 || (k >> (d == 1 ? 21 : 10)) == (cut >> (d == 1 ? 21 : 10)));
                    const int bin = (int)((k >> shift) & (unsigned)(bins - 1));
                    const unsigned long long m = __ballot(in);
                    if (m == 0ull) continue;
                    const int lead = __builtin_ctzll(m), one = __builtin_amdgcn_readlane(bin, lead);
                    if (__ballot(in && bin != one) == 0ull) {
                        if (lane == lead) atomicAdd(&hist[d][one], __popcll(m));
                    } else if (in) {
                        atomicAdd(&hist[d][bin], 1);
                    }
                }
            });
            __syncthreads();
            // suffix sums: thread i holds bins (from the top) i * PER ..; the bin in which
            // the count from the top reaches `left`
            const int per = bins / NT;
            int c[kBins / NT], sum = 0;
            #pragma unroll
            for (int i = 0; i < kBins / NT; ++i) {
                c[i] = i < per ? hist[d][bins - 1 - (tid * per + i)] : 0;
                sum += c[i];
            }
            int run = wave_prefix(sum);
            if (lane == kWave - 1) part[1 + d][wave] = run;
            __syncthreads();
            #pragma unroll
            for (int v = 0; v < NW; ++v)
                if (v < wave) run += part[1 + d][v];
            int before = run - sum;
            #pragma unroll
            for (int i = 0; i < kBins / NT; ++i) {
                if (i < per && before < left && before + c[i] >= left) {
                    s_bin[d][0] = bins - 1 - (tid * per + i);
                    s_bin[d][1] = left - before;
                }
                before += c[i];
            }
            __syncthreads();
            cut |= (unsigned int)s_bin[d][0] << shift;
            left = s_bin[d][1];
        }
    }

    // The lists, in slot order. A lane's slots are neighbours, a load's slots follow the
    // lane order and a wave's loads each other. First the ties before each slot ...
    int ties = 0;
    auto is_tie = [&](int t, int e, const float (&x)[4], unsigned int r) {
        return want > 0 && t + e >= fixed && t + e < L && (((r ^ flip) >> e) & 1u) && order_key(x[e]) == cut;
    };
    each([&](int t, const float (&x)[4], unsigned int r) {
        #pragma unroll
        for (int e = 0; e < 4; ++e) ties += is_tie(t, e, x, r);
    });
    ties = wave_sum(ties);
    __syncthreads();                     // part[0] has been read
    if (lane == 0) part[0][wave] = ties;
    __syncthreads();
    int tie0 = 0;
    #pragma unroll
    for (int v = 0; v < NW; ++v)
        if (v < wave) tie0 += part[0][v];
    // ... then who stays, twice: counted, and listed behind the counts of the waves before
    int32_t *holes = p.moves + base, *from = holes + T / 2;
    int nh = 0, ns = 0;
    auto pass = [&](auto emit) {
        int tie = tie0;
        each([&](int t, const float (&x)[4], unsigned int r) {
            int mine = 0;
            #pragma unroll
            for (int e = 0; e < 4; ++e) mine += is_tie(t, e, x, r);
            const int incl = wave_prefix(mine);
            int rank = tie + incl - mine;
            tie += __builtin_amdgcn_readlane(incl, kWave - 1);
            unsigned int hole = 0u, src = 0u;
            #pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int s = t + e;
                bool stay = s < fixed;
                if (s >= fixed && s < L) {
                    if (((r ^ flip) >> e) & 1u) {
                        const unsigned int k = order_key(x[e]);
                        stay = want > 0 && (k > cut || (k == cut && rank++ < left));
                    } else {
                        stay = !cut_recent;          // the other kind: recent ones all stay, or none of the others
                    }
                }
                if (s < keep && !stay) hole |= 1u << e;
                if (s >= keep && s < L && stay) src |= 1u << e;
            }
            emit(t, hole, src);
        });
    };
    pass([&](int, unsigned int hole, unsigned int src) {
        nh += __popc(hole);
        ns += __popc(src);
    });
    nh = wave_sum(nh);
    ns = wave_sum(ns);
    if (lane == 0) { part[1][wave] = nh; part[2][wave] = ns; }
    __syncthreads();
    int h0 = 0, s0 = 0, total = 0;
    #pragma unroll
    for (int v = 0; v < NW; ++v) {
        if (v < wave) { h0 += part[1][v]; s0 += part[2][v]; }
        total += part[1][v];
    }
    pass([&](int t, unsigned int hole, unsigned int src) {
        const int mine = __popc(hole) | (__popc(src) << 16);
        const int incl = wave_prefix(mine);
        int h = h0 + ((incl - mine) & 0xFFFF), s = s0 + ((incl - mine) >> 16);
        const int all = __builtin_amdgcn_readlane(incl, kWave - 1);
        h0 += all & 0xFFFF;
        s0 += all >> 16;
        #pragma unroll
        for (int e = 0; e < 4; ++e) {
            if ((hole >> e) & 1u) holes[h++] = t + e;
            if ((src >> e) & 1u) from[s++] = t + e;
        }
    });
    if (tid == 0) *count = p.move_here ? 0 : total;
    if (p.move_here) {
        __syncthreads();
        move_rows(p, b, g, total, tid, NT);
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
    const int g = blockIdx.y, b = blockIdx.z;
    move_rows(p, b, g, p.count[(size_t)b * p.Hkv + g], blockIdx.x * kMoveThreads + threadIdx.x,
              gridDim.x * kMoveThreads);
}

}  // namespace

hipError_t launch_evict(EvictParams p, hipStream_t s) {
    auto aligned = [](const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
    const long T = (long)p.max_pages << p.p_shift;
    p.vector_slots = T % 4 == 0 && aligned(p.weight) && aligned(p.position);
    // rows that may move: those past the kept length, into slots below it (with more
    // fixed slots than the budget none does)
    const int past = p.max_keys > p.budget ? p.max_keys - p.budget : 0;
    const int moves = past < p.budget ? past : p.budget;
    p.move_here = moves <= kFewMoves;
    const dim3 grid(p.Hkv, p.B);
    const hipError_t e =
        p.max_keys <= kSlots<256, 1>    ? launch_kernel(evict_select_kernel<256, 1>, grid, dim3(256), s, p)
        : p.max_keys <= kSlots<1024, 1> ? launch_kernel(evict_select_kernel<1024, 1>, grid, dim3(1024), s, p)
        : p.max_keys <= kSlots<1024, 4> ? launch_kernel(evict_select_kernel<1024, 4>, grid, dim3(1024), s, p)
                                        : launch_kernel(evict_select_kernel<1024, 8>, grid, dim3(1024), s, p);
    if (e != hipSuccess || p.move_here) return e;
    const long pieces = ((long)moves * p.D / 8 + kMoveThreads - 1) / kMoveThreads;
    const long per = 16384 / ((long)p.Hkv * p.B) + 1;
    return launch_kernel(evict_move_kernel, dim3((unsigned)(pieces < per ? pieces : per), p.Hkv, p.B),
                         dim3(kMoveThreads), s, p);
}

}  // namespace tv
