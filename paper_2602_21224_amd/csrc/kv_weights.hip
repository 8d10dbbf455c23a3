// Accumulated attention weight of every cached key, for gfx950.
//
// Per sequence b, KV head g and cached position t the accepted path's query
// rows (path node j, head h of g) add exp(scale * q.k_t - lse[j, h]), the
// softmax weight that the row gave the key; the rows' own keys (positions
// kv_len .. kv_len + accept_len - 1, visible to the rows at or behind them)
// get their first weight. One thread owns one key, so nothing is summed
// across threads and the order of the sums is fixed.
#include "tv_internal.h"

namespace tv {
namespace {

constexpr int kThreads = 256;

template <int D>
__global__ __launch_bounds__(kThreads) void accumulate_weights_kernel(WeightParams p) {
    const int b = blockIdx.z, g = blockIdx.y;
    const int T = p.max_pages << p.p_shift;
    const int L = min(max(p.kv_len[b], 0), T);
    const int n = min(max(p.accept_len[b], 0), p.N);
    const int fixed = p.fixed_len ? min(max(p.fixed_len[b], 0), L) : 0;
    const int end = (int)min((long long)L + n, (long long)T);
    const int G = p.Hq / p.Hkv;
    const size_t base = ((size_t)b * p.Hkv + g) * T;
    for (int t = blockIdx.x * kThreads + threadIdx.x; t < end; t += gridDim.x * kThreads) {
        if (t < fixed) {
            p.weight_out[base + t] = p.weight[base + t];
            continue;
        }
        const int pg = p.page_table[(size_t)b * p.max_pages + (t >> p.p_shift)];
        if (pg < 0 || pg >= p.num_pages) continue;
        const bf16x8 *kr = reinterpret_cast<const bf16x8 *>(
            p.k_cache + ((((size_t)pg << p.p_shift) + (t & ((1 << p.p_shift) - 1))) * p.Hkv + g) * D);
        bf16x8 k[D / 8];
        #pragma unroll
        for (int i = 0; i < D / 8; ++i) k[i] = kr[i];
        float mass = 0.f;
        for (int j = max(t - L, 0); j < n; ++j) {
            const int node = p.accept_idx[(size_t)b * p.N + j];
            if (node < 0 || node >= p.N) continue;
            for (int h = g * G; h < g * G + G; ++h) {
                const size_t row = ((size_t)b * p.N + node) * p.Hq + h;
                const float lse = p.lse[row];
                if (lse == -__builtin_huge_valf()) continue;
                const bf16x8 *qr = reinterpret_cast<const bf16x8 *>(p.q + row * D);
                float s = 0.f;
                #pragma unroll
                for (int i = 0; i < D / 8; ++i)
                    #pragma unroll
                    for (int e = 0; e < 8; ++e) s += (float)qr[i][e] * (float)k[i][e];
                mass += expf(s * p.scale - lse);
            }
        }
        p.weight_out[base + t] = t < L ? p.weight[base + t] + mass : mass;
        if (t >= L) p.position[base + t] = p.seen[b] + (t - L);
    }
}

}  // namespace

hipError_t launch_accumulate_weights(const WeightParams &p, int head_dim, hipStream_t s) {
    const long tiles = ((long)p.max_keys + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(tiles < 65535 ? tiles : 65535), p.Hkv, p.B);
    return head_dim == 64 ? launch_kernel(accumulate_weights_kernel<64>, grid, dim3(kThreads), s, p)
                          : launch_kernel(accumulate_weights_kernel<128>, grid, dim3(kThreads), s, p);
}

}  // namespace tv
