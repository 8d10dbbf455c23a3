// Tree-masked attention for batches whose sequences share a long prefix, for
// gfx950: the plain form, one wave per (sequence, node, query head), 64 keys at
// a time with one pass over them (running maximum and sum).
#include "tv_internal.h"

namespace tv {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();

template <int D>
__global__ __launch_bounds__(kWave) void shared_attention_kernel(AttnParams p) {
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z, lane = threadIdx.x;
    const int g = h / p.G;
    const size_t row = ((size_t)b * p.N + i) * p.Hq + h;
    const int nodes = p.num_nodes ? min(max(p.num_nodes[b], 0), p.N) : p.N;
    if (i >= nodes) {
        if (lane < D / 8) reinterpret_cast<u16x8 *>(p.out + row * D)[lane] = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
        if (p.lse && lane == 0) p.lse[row] = kNegInf;
        return;
    }
    const int cap = p.max_pages << p.p_shift;
    const int L = min(max(p.kv_len[b], 0), cap);
    __shared__ int path[kMaxNodes];
    int depth = 0;
    for (int j = i; j >= 0;) {
        if (lane == 0) path[depth] = j;
        ++depth;
        const int pj = p.parent[(size_t)b * p.N + j];
        j = pj < -1 || pj >= j ? -1 : pj;
    }
    __syncthreads();
    bf16x8 q[D / 8];
    #pragma unroll
    for (int c = 0; c < D / 8; ++c) q[c] = reinterpret_cast<const bf16x8 *>(p.q + row * D)[c];
    float m = kNegInf, l = 0.f, o[D / kWave] = {};
    for (int t0 = 0; t0 < L + depth; t0 += kWave) {
        const int t = t0 + lane;
        const uint16_t *kr = nullptr, *vr = nullptr;
        if (t < L) {
            const int pg = p.page_table[(size_t)b * p.max_pages + (t >> p.p_shift)];
            if (pg >= 0 && pg < p.num_pages) {
                const size_t off = ((((size_t)pg << p.p_shift) + (t & (p.P - 1))) * p.Hkv + g) * D;
                kr = p.k_cache + off;
                vr = p.v_cache + off;
            }
        } else if (t < L + depth) {
            const size_t off = (((size_t)b * p.N + path[t - L]) * p.Hkv + g) * D;
            kr = p.k_tree + off;
            vr = p.v_tree + off;
        }
        float s = kNegInf;
        if (kr) {
            s = 0.f;
            #pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const bf16x8 k = reinterpret_cast<const bf16x8 *>(kr)[c];
                #pragma unroll
                for (int e = 0; e < 8; ++e) s += (float)q[c][e] * (float)k[e];
            }
            s *= p.scale;
        }
        float mt = s;
        #pragma unroll
        for (int off = 32; off > 0; off >>= 1) mt = fmaxf(mt, __shfl_xor(mt, off));
        const float mn = fmaxf(m, mt);
        const float alpha = m == kNegInf ? 0.f : expf(m - mn);
        const float x = s == kNegInf ? 0.f : expf(s - mn);
        l = l * alpha + x;
        #pragma unroll
        for (int c = 0; c < D / kWave; ++c) o[c] *= alpha;
        m = mn;
        for (int k = 0; k < min(kWave, L + depth - t0); ++k) {
            const uint16_t *v = (const uint16_t *)__shfl((unsigned long long)vr, k);
            const float xk = __shfl(x, k);
            if (!v) continue;
            #pragma unroll
            for (int c = 0; c < D / kWave; ++c)
                o[c] += xk * (float)__builtin_bit_cast(__bf16, v[lane + c * kWave]);
        }
    }
    #pragma unroll
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off);
    #pragma unroll
    for (int c = 0; c < D / kWave; ++c)
        p.out[row * D + lane + c * kWave] = __builtin_bit_cast(uint16_t, (__bf16)(o[c] / l));
    if (p.lse && lane == 0) p.lse[row] = m + logf(l);
}

}  // namespace

hipError_t launch_shared_attention(const AttnParams &p, int head_dim, hipStream_t s) {
    const dim3 grid(p.Hq, p.N, p.B);
    return head_dim == 64 ? launch_kernel(shared_attention_kernel<64>, grid, dim3(kWave), s, p)
                          : launch_kernel(shared_attention_kernel<128>, grid, dim3(kWave), s, p);
}

}  // namespace tv
