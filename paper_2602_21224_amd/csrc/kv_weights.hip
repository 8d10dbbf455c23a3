// Accumulated attention weight of every cached key, for gfx950.
//
// Per sequence b, KV head g and cached position t the accepted path's query
// rows (path node j, head h of g) add exp(scale * q.k_t - lse[j, h]), the
// softmax weight that the row gave the key; the rows' own keys (positions
// kv_len .. kv_len + accept_len - 1, visible to the rows at or behind them)
// get their first weight.
//
// Few rows meet many keys, so the call is bound by reading K once. A wave
// holds 64 keys in registers (16-byte loads straight from the pages: the
// fragments of v_mfma_f32_16x16x32_bf16 with the keys on N, lane l holding key
// l % 16 of each of four blocks and head-dim columns 8 (l / 16) + 32 step) and
// takes the rows 16 at a time on M: lane l then holds the scores of rows
// 4 (l / 16) + i with its key, and adds their exponentials into one number per
// key block. The page ids of a wave's keys are fetched together and its keys all
// issued before anything waits for them; meanwhile the workgroup puts what the
// rows need (place of the query, log-sum-exp, last visible key) into LDS. The
// sums run over the rows in order and over l / 16 at the end: fixed, without
// atomics.
//
// Kernel times: 4 sequences x 8 KV heads of 32768 keys of 128, paths of up to 12 nodes x 4
// heads, 60-63 us (277 MB, 4.4-4.6 TB/s; a large copy reads and writes 4.8); 16 sequences
// of 1024-4096 keys 21-29 us (87 MB at their mean length), where one workgroup's wait for
// page ids, then keys, then stores is a good part of the call; 8 heads of 128 keys 4 us.
// A kernel with one thread per key took 296, 168 and 12; the same tiles with the keys
// asked for one block at a time 76 and 31.
#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;                // per wave
constexpr int kMaxRows = 2048;           // query rows per KV head (path nodes x heads of the group)
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;

template <int D>
__global__ __launch_bounds__(kThreads) void accumulate_weights_kernel(WeightParams p) {
    constexpr int NKS = D / 32;          // MFMA steps over the head dim
    // per path row: its query's offset in 16-byte pieces, its log-sum-exp in base 2, and
    // the last position it sees (-1: the row adds nothing)
    __shared__ int s_q[kMaxRows];
    __shared__ __attribute__((aligned(16))) float s_z[kMaxRows];
    __shared__ __attribute__((aligned(16))) int s_last[kMaxRows];
    const int b = blockIdx.z, g = blockIdx.y;
    const int lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int T = p.max_pages << p.p_shift;
    const int L = min(max(p.kv_len[b], 0), T);
    const int n = min(max(p.accept_len[b], 0), p.N);
    const int fixed = p.fixed_len ? min(max(p.fixed_len[b], 0), L) : 0;
    const int end = min(L + n, T);
    constexpr int kStep = kThreads / kWave * kKeys;
    if ((int)blockIdx.x * kStep >= end) return;
    const int G = p.Hq / p.Hkv;
    const int rows = n * G, padded = (rows + 15) & ~15;
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    const int32_t *table = p.page_table + (size_t)b * p.max_pages;
    const int mask = (1 << p.p_shift) - 1;
    const float c = p.scale * kLog2e;
    const uint16_t *qb = p.q + ((size_t)b * p.N * p.Hq + g * G) * D + quad * 8;

    int t0 = blockIdx.x * kStep + wave * kKeys;
    bf16x8 k[4][NKS];
    bool ok[4];
    // the wave's keys; one without a row in the pool reads the pool's first row and is
    // not written
    auto load_pages = [&](int (&pg)[4]) {
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb) pg[kb] = table[min(t0 + kb * 16 + col, T - 1) >> p.p_shift];
    };
    auto load_keys = [&](const int (&pg)[4]) {
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            const int t = t0 + kb * 16 + col;
            ok[kb] = t < end && (unsigned)pg[kb] < (unsigned)p.num_pages;
            const size_t slot = ok[kb] ? ((size_t)pg[kb] << p.p_shift) + (t & mask) : 0;
            const uint16_t *kr = p.k_cache + (slot * p.Hkv + g) * D + quad * 8;
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                k[kb][ks] = *reinterpret_cast<const bf16x8 *>(kr + ks * 32);
        }
    };
    const bool work = t0 < end && t0 + kKeys > fixed;
    // The first rows' node ids and log-sum-exps are asked for before the keys, which loads
    // return in order: waiting for them then does not wait for the keys.
    int pages[4] = {0, 0, 0, 0};
    if (work) load_pages(pages);
    int j, nd, at;
    float z = 0.f;
    auto ask = [&](int r) {
        const int x = min(r, rows - 1);
        j = p.g_inv ? (int)__umulhi((unsigned)x, p.g_inv) : x;
        nd = p.accept_idx[(size_t)b * p.N + j];
        at = min(max(nd, 0), p.N - 1) * p.Hq + (x - j * G);
        z = p.lse[(size_t)b * p.N * p.Hq + g * G + at];
    };
    int r = threadIdx.x;
    if (r < padded) ask(r);
    if (work) load_keys(pages);
    while (r < padded) {
        const bool real = r < rows && (unsigned)nd < (unsigned)p.N && z != kNegInf;
        s_q[r] = at * (D / 8);
        s_z[r] = z * kLog2e;
        s_last[r] = real ? L + j : -1;
        r += kThreads;
        if (r < padded) ask(r);
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");

    for (bool again = false; t0 < end; t0 += gridDim.x * kStep, again = true) {
        const int mine = t0 + lane;      // the key whose weight this lane writes
        if (t0 + kKeys <= fixed) {
            if (p.weight_out != p.weight) p.weight_out[base + mine] = p.weight[base + mine];
            continue;
        }
        if (again) {
            load_pages(pages);
            load_keys(pages);
        }
        const float old = mine < L ? p.weight[base + mine] : 0.f;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        bf16x8 q[2][NKS];
        auto load_q = [&](int r0, bf16x8 (&x)[NKS]) {
            const uint16_t *qr = qb + (size_t)s_q[r0 + col] * 8;
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks) x[ks] = *reinterpret_cast<const bf16x8 *>(qr + ks * 32);
        };
        auto block = [&](int r0, const bf16x8 (&x)[NKS]) {
            const f32x4 z = *reinterpret_cast<const f32x4 *>(s_z + r0 + 4 * quad);
            const i32x4 last = *reinterpret_cast<const i32x4 *>(s_last + r0 + 4 * quad);
            #pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int ks = 0; ks < NKS; ++ks)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[ks], k[kb][ks], s, 0, 0, 0);
                const int t = t0 + kb * 16 + col;
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -z[i]));
                    sum[kb] += t <= last[i] ? e : 0.f;
                }
            }
        };
        // 16 rows at a time on M (lane l loads row l % 16), the next ones on their way
        if (padded > 0) load_q(0, q[0]);
        for (int r0 = 0; r0 < padded; r0 += 32) {
            if (r0 + 16 < padded) load_q(r0 + 16, q[1]);
            block(r0, q[0]);
            if (r0 + 32 < padded) load_q(r0 + 32, q[0]);
            if (r0 + 16 < padded) block(r0 + 16, q[1]);
        }
        // over the four row groups; lane l then takes key block l / 16
        float total = 0.f;
        bool live = false;
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            float x = sum[kb];
            x += __shfl_xor(x, 16);
            x += __shfl_xor(x, 32);
            if (quad == kb) {
                total = x;
                live = ok[kb];
            }
        }
        if (mine >= end) continue;
        if (mine < fixed) {
            if (p.weight_out != p.weight) p.weight_out[base + mine] = old;
        } else if (live) {
            p.weight_out[base + mine] = old + total;
            if (mine >= L) p.position[base + mine] = p.seen[b] + (mine - L);
        }
    }
}

}  // namespace

hipError_t launch_accumulate_weights(const WeightParams &p, int head_dim, hipStream_t s) {
    constexpr int kPerWg = kThreads / kWave * kKeys;
    const long tiles = ((long)p.max_keys + kPerWg - 1) / kPerWg;
    const dim3 grid((unsigned)(tiles < 65535 ? tiles : 65535), p.Hkv, p.B);
    return head_dim == 64 ? launch_kernel(accumulate_weights_kernel<64>, grid, dim3(kThreads), s, p)
                          : launch_kernel(accumulate_weights_kernel<128>, grid, dim3(kThreads), s, p);
}

}  // namespace tv
