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
// key block. Nothing goes through LDS, and waves need no barrier. The sums run
// over the rows in order and over l / 16 at the end: fixed, without atomics.
#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;                // per wave
constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f;

template <int D>
__global__ __launch_bounds__(kThreads) void accumulate_weights_kernel(WeightParams p) {
    constexpr int NKS = D / 32;          // MFMA steps over the head dim
    const int b = blockIdx.z, g = blockIdx.y;
    const int lane = threadIdx.x & (kWave - 1), col = lane & 15, quad = lane >> 4;
    const int T = p.max_pages << p.p_shift;
    const int L = min(max(p.kv_len[b], 0), T);
    const int n = min(max(p.accept_len[b], 0), p.N);
    const int fixed = p.fixed_len ? min(max(p.fixed_len[b], 0), L) : 0;
    const int end = min(L + n, T);
    const int G = p.Hq / p.Hkv;
    const int rows = n * G;
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    const int32_t *table = p.page_table + (size_t)b * p.max_pages;
    const int32_t *path = p.accept_idx + (size_t)b * p.N;
    const int mask = (1 << p.p_shift) - 1;
    const float c = p.scale * kLog2e;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int step = gridDim.x * (kThreads / kWave) * kKeys;
    for (int t0 = (blockIdx.x * (kThreads / kWave) + wave) * kKeys; t0 < end; t0 += step) {
        const int mine = t0 + lane;      // the key whose weight this lane writes
        if (t0 + kKeys <= fixed) {
            if (p.weight_out != p.weight) p.weight_out[base + mine] = p.weight[base + mine];
            continue;
        }
        // the wave's keys; one without a row in the pool reads the pool's first row and
        // is not written
        bf16x8 k[4][NKS];
        bool ok[4];
        #pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            const int t = t0 + kb * 16 + col;
            const int pg = t < end ? table[t >> p.p_shift] : -1;
            ok[kb] = pg >= 0 && pg < p.num_pages;
            const size_t slot = ok[kb] ? ((size_t)pg << p.p_shift) + (t & mask) : 0;
            const uint16_t *kr = p.k_cache + (slot * p.Hkv + g) * D + quad * 8;
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                k[kb][ks] = *reinterpret_cast<const bf16x8 *>(kr + ks * 32);
        }
        const float old = mine < L ? p.weight[base + mine] : 0.f;

        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r0 = 0; r0 < rows; r0 += 16) {
            // Q rows on M: lane l loads row l % 16 (a row past the last one, or of a node
            // out of range, loads node 0's and counts for nothing)
            const int rq = r0 + col, jq = rq / G;
            int nq = rq < rows ? path[jq] : 0;
            if (nq < 0 || nq >= p.N) nq = 0;
            const uint16_t *qr =
                p.q + (((size_t)b * p.N + nq) * p.Hq + g * G + (rq - jq * G)) * D + quad * 8;
            bf16x8 q[NKS];
            #pragma unroll
            for (int ks = 0; ks < NKS; ++ks) q[ks] = *reinterpret_cast<const bf16x8 *>(qr + ks * 32);
            // the rows whose scores this lane gets: their lse, and the last key they see
            float z[4];
            int last[4];
            #pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + 4 * quad + i, j = r / G;
                const int nd = r < rows ? path[j] : -1;
                const bool real = nd >= 0 && nd < p.N;
                const float l = real ? p.lse[((size_t)b * p.N + nd) * p.Hq + g * G + (r - j * G)] : kNegInf;
                z[i] = l * kLog2e;
                last[i] = l == kNegInf ? -1 : L + j;
            }
            #pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
                #pragma unroll
                for (int ks = 0; ks < NKS; ++ks)
                    s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[ks], k[kb][ks], s, 0, 0, 0);
                const int t = t0 + kb * 16 + col;
                #pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -z[i]));
                    sum[kb] += t <= last[i] ? x : 0.f;
                }
            }
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
