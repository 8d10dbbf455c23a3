// Eviction from the paged cache by accumulated attention weight, for gfx950.
//
// The slots of a (sequence, KV head) fall into three kinds that rank before
// one another (fixed, recent, others); the budget cuts one of the last two,
// and there the cut is the k-th largest weight. One workgroup per (sequence,
// KV head) finds it:
//   * Every wave owns one run of slots and holds their order-preserving 32-bit
//     keys in registers (four neighbouring slots per lane and load), so the
//     passes below read nothing again; caches of more slots per head than the
//     largest instance holds re-read theirs (L2) in the same passes.
//   * Radix select in digits of 11, 11 and 10 bits. The first histogram takes
//     every key (a lane adds a run of equal digits once, so that equal weights do
//     not serialise); the keys of the bin that holds the cut, usually a few per
//     cent, are then put into a list in LDS, and the other two digits only look
//     at that. A bin is found by a suffix sum over all threads (a scan within the
//     wave by DPP, one exchange between the waves).
//   * Among the keys equal to the cut the lowest slots stay; they are counted
//     only if not all of them stay. Who is evicted below the kept length and who
//     is kept past it is noted in two bit masks per lane, and one exchange of the
//     waves' counts gives each wave its place in the two lists of slots, which
//     come out in slot order.
// The k-th slot of the first list takes the row of the k-th of the second:
// sources lie past the kept length and destinations below it, so no move reads
// what another wrote, and only rows that have to move do. A second kernel moves
// them with the whole chip; where there can be few, the first does.
//
// Kernel times: 4 sequences x 8 KV heads from 32768 slots to 8192, 27 us of selection (one
// workgroup's passes over its registers; 32 CUs read 8 MB) and 43-45 us of moves (195 MB
// in and out, 4.4 TB/s); 16 x 8 heads of 1900-2311 slots to 2048 11.6 us in one
// kernel; 8 heads of 128 slots 7 us, a chain of barriers. A selection that re-read its
// weights for every 8-bit digit and moved its rows itself took 447, 48 and 34.
#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kBins = 2048;
constexpr int kList = 4096;         // keys of the cut's bin that are looked at in LDS
constexpr int kMoveThreads = 256;
constexpr int kFewPieces = 8;       // 16-byte pieces (of K and of V) per thread that the selecting workgroup moves itself

// Slots in registers: ITER loads of 4 per lane.
template <int NT, int ITER>
constexpr int kSlots = NT * 4 * ITER;

__device__ __forceinline__ int wave_sum(int x) {
    return __builtin_amdgcn_readlane(wave_prefix_sum(x), kWave - 1);
}
// Set bits, of four per lane, in the lanes before this one, and in all of them.
__device__ __forceinline__ int bits_before(unsigned int nibble, int &all) {
    int n = 0;
    all = 0;
    #pragma unroll
    for (int e = 0; e < 4; ++e) {
        const unsigned long long m = __ballot((nibble >> e) & 1u);
        n = __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, n));
        all += __popcll(m);
    }
    return n;
}

// Moves of one (sequence, KV head): threads tid, tid + step, ... of all that share
// them take 16-byte pieces of the rows' K and V, U at a time so that the chains of
// loads (slots, page ids, rows) of U pieces run side by side.
template <int U>
__device__ __forceinline__ void move_rows(const EvictParams &p, int b, int g, int n, int tid, int step) {
    const int T = p.max_pages << p.p_shift;
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    const int32_t *holes = p.moves + base, *from = holes + T / 2;
    const int32_t *table = p.page_table + (size_t)b * p.max_pages;
    const int chunks = p.D / 8, mask = (1 << p.p_shift) - 1;
    const int pieces = n * chunks;
    for (int i0 = tid; i0 < pieces; i0 += U * step) {
        int dst[U], src[U], c[U], pd[U], ps[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            // a piece past the last one repeats it, and is not stored
            const int i = min(i0 + u * step, pieces - 1);
            const int m = p.chunk_shift >= 0 ? i >> p.chunk_shift : i / chunks;
            c[u] = i - m * chunks;
            dst[u] = holes[m];
            src[u] = from[m];
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            pd[u] = table[dst[u] >> p.p_shift];
            ps[u] = table[src[u] >> p.p_shift];
        }
        u16x8 k[U], v[U];
        float w[U];
        int y[U];
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool ok = (unsigned)pd[u] < (unsigned)p.num_pages && (unsigned)ps[u] < (unsigned)p.num_pages;
            const size_t slot = ok ? ((size_t)ps[u] << p.p_shift) + (src[u] & mask) : 0;
            const size_t at = (slot * p.Hkv + g) * p.D + c[u] * 8;
            k[u] = *reinterpret_cast<const u16x8 *>(p.k_cache + at);
            v[u] = *reinterpret_cast<const u16x8 *>(p.v_cache + at);
            if (!ok) pd[u] = -1;
            if (c[u] == 0) {
                w[u] = p.weight[base + src[u]];
                y[u] = p.position[base + src[u]];
            }
        }
        #pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * step >= pieces) continue;
            if (c[u] == 0) {
                p.weight_out[base + dst[u]] = w[u];
                p.position_out[base + dst[u]] = y[u];
            }
            if (pd[u] < 0) continue;
            const size_t at = ((((size_t)pd[u] << p.p_shift) + (dst[u] & mask)) * p.Hkv + g) * p.D + c[u] * 8;
            *reinterpret_cast<u16x8 *>(p.k_cache + at) = k[u];
            *reinterpret_cast<u16x8 *>(p.v_cache + at) = v[u];
        }
    }
}

template <int NT, int ITER>
__global__ __launch_bounds__(NT) void evict_select_kernel(EvictParams p) {
    static_assert(ITER <= 8, "a lane's slots are bits of one word");
    constexpr int NW = NT / kWave;
    __shared__ int hist[3][kBins];
    __shared__ unsigned int list[kList];
    __shared__ int part[7][NW];
    __shared__ int s_bin[3][3];
    __shared__ int s_listed;
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
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
    // Bit e: slot t + e lies in [lo, hi).
    auto within = [](int t, int lo, int hi) {
        const int a = min(max(lo - t, 0), 4), c = min(max(hi - t, 0), 4);
        return ((1u << c) - 1u) & ~((1u << a) - 1u);
    };
    auto recent_of = [&](int t, const int (&y)[4]) {
        unsigned int r = 0u;
        #pragma unroll
        for (int e = 0; e < 4; ++e) r |= (y[e] >= newest ? 1u : 0u) << e;
        return r & within(t, fixed, L);
    };
    unsigned int key[ITER][4];
    unsigned int recent = 0u;            // bit 4 i + e: slot e of load i is a recent one
    // `body(i, t, k, r)` over this lane's slots: t the first of four, k their keys, r the
    // bits of the recent ones
    auto each = [&](auto body) {
        if (held) {
            #pragma unroll
            for (int i = 0; i < ITER; ++i)
                if (i < iters) body(i, first + i * 4 * kWave, key[i], (recent >> (4 * i)) & 15u);
        } else {
            for (int i = 0; i < iters; ++i) {
                const int t = first + i * 4 * kWave;
                float x[4];
                int y[4];
                load(t, x, y);
                unsigned int k[4];
                #pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = order_key(x[e]);
                body(0, t, k, recent_of(t, y));
            }
        }
    };

    // weights and positions, once; arrays of their own take what may stay where it is
    // (slots that are evicted are written again by their moves)
    int recents = 0;
    auto copy_out = [&](int t, const float (&x)[4], const int (&y)[4]) {
        if (p.vector_out && t + 4 <= keep) {
            if (wout) *reinterpret_cast<f32x4 *>(wout + t) = f32x4{x[0], x[1], x[2], x[3]};
            if (pout) *reinterpret_cast<i32x4 *>(pout + t) = i32x4{y[0], y[1], y[2], y[3]};
            return;
        }
        #pragma unroll
        for (int e = 0; e < 4; ++e)
            if (t + e < keep) {
                if (wout) wout[t + e] = x[e];
                if (pout) pout[t + e] = y[e];
            }
    };
    if (held) {
        float x[ITER][4];
        int y[ITER][4];
        #pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (i < iters) load(first + i * 4 * kWave, x[i], y[i]);
        #pragma unroll
        for (int i = 0; i < 3 * kBins / NT; ++i) hist[(i * NT + tid) / kBins][(i * NT + tid) % kBins] = 0;
        if (tid == 0) s_listed = 0;
        #pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (i < iters) {
                const int t = first + i * 4 * kWave;
                #pragma unroll
                for (int e = 0; e < 4; ++e) key[i][e] = order_key(x[i][e]);
                recent |= recent_of(t, y[i]) << (4 * i);
                if (wout || pout) copy_out(t, x[i], y[i]);
            }
        recents = __popc(recent);
    } else {
        for (int i = tid; i < 3 * kBins; i += NT) hist[i / kBins][i % kBins] = 0;
        if (tid == 0) s_listed = 0;
        for (int i = 0; i < iters; ++i) {
            const int t = first + i * 4 * kWave;
            float x[4];
            int y[4];
            load(t, x, y);
            recents += __popc(recent_of(t, y));
            if (wout || pout) copy_out(t, x, y);
        }
    }
    if (keep == L) {
        if (tid == 0) *count = 0;
        return;
    }
    // The waves' counts behind one another: sum of those before this wave, and of all.
    auto exchange = [&](int row, int x, int &all) {
        if (lane == 0) part[row][wave] = x;
        __syncthreads();
        int before = 0;
        all = 0;
        #pragma unroll
        for (int v = 0; v < NW; ++v) {
            const int y = part[row][v];
            before += v < wave ? y : 0;
            all += y;
        }
        return before;
    };
    int total;
    exchange(0, wave_sum(recents), total);
    recents = total;

    // which kind the budget cuts, and how many of it stay
    const bool cut_recent = recents >= keep - fixed;
    const int want = cut_recent ? keep - fixed : keep - fixed - recents;
    const unsigned int flip = cut_recent ? 0u : 15u;
    auto cut_kind = [&](int t, unsigned int r) { return (r ^ flip) & within(t, fixed, L); };
    unsigned int cut = 0u;
    int left = want, equal = 0;          // of the `equal` keys at the cut, how many stay
    // The bin of digit d in which the count from the top reaches `left`: thread i holds bins
    // (from the top) i * per ..
    auto find = [&](int d, int shift, int bins) {
        __syncthreads();
        const int per = bins / NT;
        int c[kBins / NT], sum = 0;
        #pragma unroll
        for (int i = 0; i < kBins / NT; ++i) {
            c[i] = i < per ? hist[d][bins - 1 - (tid * per + i)] : 0;
            sum += c[i];
        }
        const int incl = wave_prefix_sum(sum);
        int all;
        int before = exchange(1 + d, __builtin_amdgcn_readlane(incl, kWave - 1), all) + incl - sum;
        #pragma unroll
        for (int i = 0; i < kBins / NT; ++i) {
            if (i < per && before < left && before + c[i] >= left) {
                s_bin[d][0] = bins - 1 - (tid * per + i);
                s_bin[d][1] = left - before;
                s_bin[d][2] = c[i];
            }
            before += c[i];
        }
        __syncthreads();
        cut |= (unsigned int)s_bin[d][0] << shift;
        left = s_bin[d][1];
        equal = s_bin[d][2];
    };
    // Counts a digit of the cut kind's keys whose higher digits are the cut's.
    auto histogram = [&](int d, int shift, int bins, bool all) {
        int bin = -1, run = 0;
        each([&](int, int t, const unsigned int (&k)[4], unsigned int r) {
            const unsigned int in = cut_kind(t, r);
            #pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!((in >> e) & 1u) || (!all && ((k[e] ^ cut) >> (shift + (d == 1 ? 11 : 10))) != 0u)) continue;
                const int x = (int)((k[e] >> shift) & (unsigned)(bins - 1));
                if (x != bin && run > 0) {
                    atomicAdd(&hist[d][bin], run);
                    run = 0;
                }
                bin = x;
                ++run;
            }
        });
        if (run > 0) atomicAdd(&hist[d][bin], run);
    };
    if (want > 0) {
        histogram(0, 21, 2048, true);
        find(0, 21, 2048);
        if (equal <= kList) {
            const int n = equal;
            each([&](int, int t, const unsigned int (&k)[4], unsigned int r) {
                const unsigned int in = cut_kind(t, r);
                #pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (((in >> e) & 1u) && ((k[e] ^ cut) >> 21) == 0u) list[atomicAdd(&s_listed, 1)] = k[e];
            });
            __syncthreads();
            for (int i = tid; i < n; i += NT) atomicAdd(&hist[1][(list[i] >> 10) & 2047u], 1);
            find(1, 10, 2048);
            for (int i = tid; i < n; i += NT)
                if (((list[i] ^ cut) >> 10) == 0u) atomicAdd(&hist[2][list[i] & 1023u], 1);
            find(2, 0, 1024);
        } else {
            histogram(1, 10, 2048, false);
            find(1, 10, 2048);
            histogram(2, 0, 1024, false);
            find(2, 0, 1024);
        }
    }

    // Who stays. The ties before this wave's are counted only where some of them go.
    const bool some_ties_go = want > 0 && left < equal;
    int tie0 = 0;
    if (some_ties_go) {
        int ties = 0;
        each([&](int, int t, const unsigned int (&k)[4], unsigned int r) {
            const unsigned int in = cut_kind(t, r);
            #pragma unroll
            for (int e = 0; e < 4; ++e) ties += ((in >> e) & 1u) && k[e] == cut;
        });
        tie0 = exchange(4, wave_sum(ties), total);
    }
    // Bits of the slots that are evicted below the kept length, and kept past it.
    auto judge = [&](int t, const unsigned int (&k)[4], unsigned int r, int &tie, unsigned int &hole,
                     unsigned int &src) {
        const unsigned int in = cut_kind(t, r);
        unsigned int above = 0u, at = 0u;
        #pragma unroll
        for (int e = 0; e < 4; ++e) {
            above |= (k[e] > cut ? 1u : 0u) << e;
            at |= (k[e] == cut ? 1u : 0u) << e;
        }
        at &= in;
        if (some_ties_go) {
            int all, rank = tie + bits_before(at, all);
            tie += all;
            #pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((at >> e) & 1u) {
                    if (rank >= left) at &= ~(1u << e);
                    ++rank;
                }
        }
        // the other kind: recent slots all stay, of the others none does
        const unsigned int stay = within(t, 0, fixed) | (want > 0 ? (above & in) | at : 0u) |
                                  (cut_recent ? 0u : r);
        hole = within(t, 0, keep) & ~stay;
        src = within(t, keep, L) & stay;
    };
    unsigned int holes_of = 0u, srcs_of = 0u;
    int nh = 0, ns = 0, tie = tie0;
    each([&](int i, int t, const unsigned int (&k)[4], unsigned int r) {
        unsigned int hole, src;
        judge(t, k, r, tie, hole, src);
        nh += __popc(hole);
        ns += __popc(src);
        holes_of |= hole << (4 * i);     // (of use where the slots are held)
        srcs_of |= src << (4 * i);
    });
    int32_t *holes = p.moves + base, *from = holes + T / 2;
    nh = wave_sum(nh);
    ns = wave_sum(ns);
    if (lane == 0) part[5][wave] = ns;
    int h0 = exchange(6, nh, total), s0 = 0;
    #pragma unroll
    for (int v = 0; v < NW; ++v) s0 += v < wave ? part[5][v] : 0;
    auto emit = [&](int t, unsigned int hole, unsigned int src) {
        if (__ballot(hole) != 0ull) {
            int all, h = h0 + bits_before(hole, all);
            h0 += all;
            #pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((hole >> e) & 1u) holes[h++] = t + e;
        }
        if (__ballot(src) != 0ull) {
            int all, s = s0 + bits_before(src, all);
            s0 += all;
            #pragma unroll
            for (int e = 0; e < 4; ++e)
                if ((src >> e) & 1u) from[s++] = t + e;
        }
    };
    if (held) {
        #pragma unroll
        for (int i = 0; i < ITER; ++i)
            if (i < iters)
                emit(first + i * 4 * kWave, (holes_of >> (4 * i)) & 15u, (srcs_of >> (4 * i)) & 15u);
    } else {
        tie = tie0;
        each([&](int, int t, const unsigned int (&k)[4], unsigned int r) {
            unsigned int hole, src;
            judge(t, k, r, tie, hole, src);
            emit(t, hole, src);
        });
    }
    if (tid == 0) *count = p.move_here ? 0 : total;
    if (p.move_here) {
        __syncthreads();
        move_rows<4>(p, b, g, total, tid, NT);
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictParams p) {
    const int g = blockIdx.y, b = blockIdx.z;
    move_rows<1>(p, b, g, p.count[(size_t)b * p.Hkv + g], blockIdx.x * kMoveThreads + threadIdx.x,
              gridDim.x * kMoveThreads);
}

}  // namespace

hipError_t launch_evict(EvictParams p, hipStream_t s) {
    auto aligned = [](const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
    const long T = (long)p.max_pages << p.p_shift;
    p.vector_slots = T % 4 == 0 && aligned(p.weight) && aligned(p.position);
    const int chunks = p.D / 8;
    p.chunk_shift = (chunks & (chunks - 1)) == 0 ? __builtin_ctz((unsigned)chunks) : -1;
    p.vector_out = p.vector_slots && aligned(p.weight_out) && aligned(p.position_out);
    // rows that may move: those past the kept length, into slots below it (with more
    // fixed slots than the budget none does)
    const int past = p.max_keys > p.budget ? p.max_keys - p.budget : 0;
    const int moves = past < p.budget ? past : p.budget;
    const int threads = p.max_keys <= kSlots<256, 1> ? 256 : 1024;
    // One launch less is worth 1 us and more; 260 rows of 128 take the selecting workgroups
    // as long as the whole chip with its launch (16 sequences x 8 heads: 11.2 us in one
    // kernel, 7.7 + 4.4 in two).
    p.move_here = (long)moves * chunks <= (long)kFewPieces * threads;
    const dim3 grid(p.Hkv, p.B), block(threads);
    const hipError_t e =
        p.max_keys <= kSlots<256, 1>    ? launch_kernel(evict_select_kernel<256, 1>, grid, block, s, p)
        : p.max_keys <= kSlots<1024, 1> ? launch_kernel(evict_select_kernel<1024, 1>, grid, block, s, p)
        : p.max_keys <= kSlots<1024, 4> ? launch_kernel(evict_select_kernel<1024, 4>, grid, block, s, p)
                                        : launch_kernel(evict_select_kernel<1024, 8>, grid, block, s, p);
    if (e != hipSuccess || p.move_here) return e;
    const long pieces = ((long)moves * p.D / 8 + kMoveThreads - 1) / kMoveThreads;
    const long per = 16384 / ((long)p.Hkv * p.B) + 1;
    return launch_kernel(evict_move_kernel, dim3((unsigned)(pieces < per ? pieces : per), p.Hkv, p.B),
                         dim3(kMoveThreads), s, p);
}

}  // namespace tv
