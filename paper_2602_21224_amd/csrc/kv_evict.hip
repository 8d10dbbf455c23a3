// Eviction from the paged cache by accumulated attention weight, for gfx950.
//
// One workgroup per (sequence, KV head). The slots fall into three kinds that
// rank before one another (fixed, recent, others); only one of the last two
// is cut by the budget, and in it the cut is the k-th largest weight, found
// by a radix select over the order-preserving 32-bit keys (four histograms of
// one byte each). Among the keys equal to the cut the lowest slots stay. A
// last pass in slot order then numbers the evicted slots below the kept
// length and the kept slots past it; the k-th of the one takes the row of the
// k-th of the other, so only rows that have to move do. Sources lie past the
// kept length and destinations below it: no move reads what another wrote.
#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / kWave;

// Sum of x over the workgroup; all threads get it. `tmp` holds one int per wave.
__device__ __forceinline__ int block_sum(int x, int *tmp) {
    #pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) tmp[threadIdx.x / kWave] = x;
    __syncthreads();
    int s = 0;
    #pragma unroll
    for (int w = 0; w < kWaves; ++w) s += tmp[w];
    return s;
}

// Threads before this one whose flag is set, over the workgroup, and the total.
__device__ __forceinline__ int block_rank(bool flag, int *tmp, int &total) {
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const unsigned long long m = __ballot(flag);
    __syncthreads();
    if (lane == 0) tmp[wave] = __popcll(m);
    __syncthreads();
    int before = __popcll(m & ((1ull << lane) - 1ull));
    total = 0;
    #pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += tmp[w];
        total += tmp[w];
    }
    return before;
}

__global__ __launch_bounds__(kThreads) void evict_kernel(EvictParams p) {
    __shared__ int hist[256];
    __shared__ int tmp[kWaves];
    __shared__ int s_cut[2];
    const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int T = p.max_pages << p.p_shift;
    const int L = min(max(p.kv_len[b], 0), T);
    const int fixed = p.fixed_len ? min(max(p.fixed_len[b], 0), L) : 0;
    const int keep = min(L, max(p.budget, fixed));
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    const float *weight = p.weight + base;
    const int32_t *position = p.position + base;
    if (g == 0 && tid == 0) p.kept_len[b] = keep;
    const long long newest = (long long)p.seen[b] - p.recent;
    if (keep == L) {
        if (p.weight_out != p.weight)
            for (int t = tid; t < keep; t += kThreads) p.weight_out[base + t] = weight[t];
        if (p.position_out != p.position)
            for (int t = tid; t < keep; t += kThreads) p.position_out[base + t] = position[t];
        return;
    }

    // which kind the budget cuts, and how many of it stay
    int mine = 0;
    for (int t = fixed + tid; t < L; t += kThreads) mine += position[t] >= newest;
    const int recents = block_sum(mine, tmp);
    const bool cut_recent = recents >= keep - fixed;
    const int want = cut_recent ? keep - fixed : keep - fixed - recents;

    // the want-th largest key of the cut kind, one byte at a time
    unsigned int cut = 0u;
    int left = want;
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int t = fixed + tid; t < L; t += kThreads) {
            if ((position[t] >= newest) != cut_recent) continue;
            const unsigned int k = order_key(weight[t]);
            if (shift == 24 || (k >> (shift + 8)) == (cut >> (shift + 8)))
                atomicAdd(&hist[(k >> shift) & 255u], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int rest = left, v = 255;
            while (v > 0 && hist[v] < rest) rest -= hist[v--];
            s_cut[0] = v;
            s_cut[1] = rest;
        }
        __syncthreads();
        cut |= (unsigned int)s_cut[0] << shift;
        left = s_cut[1];
    }

    // slots in order: evicted ones below `keep`, kept ones past it
    int32_t *holes = p.moves + base, *from = holes + T / 2;
    int ties = 0, nh = 0, ns = 0;
    for (int t0 = 0; t0 < L; t0 += kThreads) {
        const int t = t0 + tid;
        bool stay = t < fixed, tie = false;
        if (t >= fixed && t < L) {
            const bool recent = position[t] >= newest;
            const unsigned int k = order_key(weight[t]);
            if (recent != cut_recent) stay = recent;
            else if (want > 0) {
                stay = k > cut;
                tie = k == cut;
            }
        }
        int total;
        const int r = block_rank(tie, tmp, total);
        if (tie) stay = ties + r < left;
        ties += total;
        const bool hole = t < keep && !stay, src = t >= keep && t < L && stay;
        const int h = block_rank(hole, tmp, total);
        if (hole) holes[nh + h] = t;
        nh += total;
        const int s = block_rank(src, tmp, total);
        if (src) from[ns + s] = t;
        ns += total;
        if (t < keep && !hole) {
            if (p.weight_out != p.weight) p.weight_out[base + t] = weight[t];
            if (p.position_out != p.position) p.position_out[base + t] = position[t];
        }
    }
    __syncthreads();

    const int chunks = p.D / 8;
    const int mask = (1 << p.p_shift) - 1;
    const int32_t *table = p.page_table + (size_t)b * p.max_pages;
    for (int i = tid; i < ns * chunks; i += kThreads) {
        const int m = i / chunks, c = i % chunks;
        const int dst = holes[m], src = from[m];
        if (c == 0) {
            p.weight_out[base + dst] = weight[src];
            p.position_out[base + dst] = position[src];
        }
        const int pd = table[dst >> p.p_shift], ps = table[src >> p.p_shift];
        if (pd < 0 || pd >= p.num_pages || ps < 0 || ps >= p.num_pages) continue;
        const size_t d = ((((size_t)pd << p.p_shift) + (dst & mask)) * p.Hkv + g) * p.D + c * 8;
        const size_t s = ((((size_t)ps << p.p_shift) + (src & mask)) * p.Hkv + g) * p.D + c * 8;
        *reinterpret_cast<u16x8 *>(p.k_cache + d) = *reinterpret_cast<const u16x8 *>(p.k_cache + s);
        *reinterpret_cast<u16x8 *>(p.v_cache + d) = *reinterpret_cast<const u16x8 *>(p.v_cache + s);
    }
}

}  // namespace

hipError_t launch_evict(const EvictParams &p, hipStream_t s) {
    return launch_kernel(evict_kernel, dim3(p.Hkv, p.B), dim3(kThreads), s, p);
}

}  // namespace tv
