// Rows of K and V into a paged cache held in 4 bits (kv4.h), for gfx950.
//
// For every block of 32 values of a row, with amax = f 2^x, 1 <= f < 2:
//   e = x - 2 + (f > 1.75)    the smallest e with amax <= 7 2^e, within [-126, 125] (so that
//                             2^-e is a normal number, and 6 2^e a bf16)
//   code(v) = the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |v| / 2^e (ties to the even
//             code, what exceeds 6 to 6), with v's sign
// so the block's largest value is off by at most a fifth: with x - 2 throughout, one of nearly
// 8 2^e would be cut to 6 2^e, a quarter off.
//
// A workgroup takes one KV head of as many consecutive tokens as 256 threads hold (16 at
// head size 128): eight values per thread, so a block is a quad of lanes and its maximum two
// quad permutations. Tokens of one page lie together in the cache per head, so the codes
// leave as whole kilobytes; heads are the fastest index of the grid, so that the source
// rows, which lie token by token, are read by neighbours.
//
// Bound by bytes: 4 prompts of 8192 tokens (8 KV heads of 128) take 60 us, 134 MB read and 170
// MB written with the held rows, 5.1 TB/s (a copy reaches 4.8). One token takes 3 us: its
// length, its page id and its row, one after the other.
#include "kv4.h"

namespace tv {
namespace {

constexpr int kWriteThreads = 256;

__device__ __forceinline__ unsigned quad_max(unsigned x) {
    x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false));    // lanes 1 0 3 2
    return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false)); // lanes 2 3 0 1
}

// The codes of eight values of a block and (the same in its four lanes) its scale byte. A
// block that holds a NaN or an infinity, which four bits cannot, is NaN whole.
__device__ __forceinline__ unsigned to4x8(const u16x8 &x, unsigned &byte) {
    unsigned top = 0;
    #pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, (unsigned)x[i] & 0x7FFFu);
    top = quad_max(top);
    if (top >= 0x7F80u) {
        byte = 255;
        return 0;
    }
    byte = (unsigned)min(max((int)(top >> 7) - 2 + ((top & 0x7Fu) > 0x60u ? 1 : 0), 1), 252);
    const float inv = __uint_as_float((254u - byte) << 23);        // 2^-e, a normal number
    float y[8];
    #pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __uint_as_float((unsigned)x[i] << 16) * inv;
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.f, 3);
    return c;
}

template <int D>
__global__ __launch_bounds__(kWriteThreads) void kv4_write_kernel(Kv4WriteParams p) {
    constexpr int kLanes = D / 8;                          // lanes of a row
    constexpr int kTokens = kWriteThreads / kLanes;
    const int b = blockIdx.y;
    const int g = (int)(blockIdx.x % (unsigned)p.Hkv);
    const int j = (int)(blockIdx.x / (unsigned)p.Hkv) * kTokens + threadIdx.x / kLanes;
    const int n = p.count ? min(p.count[b], p.T) : p.T;
    if (j >= n) return;
    const int ln = threadIdx.x % kLanes;
    const int src = p.idx ? p.idx[(size_t)b * p.T + j] : j;
    const long pos = (long)p.start[b] + j;
    const long slot_page = pos >> p.p_shift;
    if ((unsigned)src >= (unsigned)p.T || pos < 0 || slot_page >= p.max_pages) return;
    const int pg = p.page_table[(size_t)b * p.max_pages + slot_page];
    if ((unsigned)pg >= (unsigned)p.num_pages) return;
    const size_t row = (((size_t)pg * p.Hkv + g) << p.p_shift) + (pos & ((1 << p.p_shift) - 1));
    const size_t from = (((size_t)b * p.T + src) * p.Hkv + g) * D + ln * 8;
    const size_t held = (((size_t)b * p.T + j) * p.Hkv + g) * D + ln * 8;
    const u16x8 kx = *reinterpret_cast<const u16x8 *>(p.k + from);
    const u16x8 vx = *reinterpret_cast<const u16x8 *>(p.v + from);
    unsigned ke, ve;
    const unsigned kc = to4x8(kx, ke), vc = to4x8(vx, ve);
    *reinterpret_cast<unsigned *>(p.k4 + row * (D / 2) + ln * 4) = kc;
    *reinterpret_cast<unsigned *>(p.v4 + row * (D / 2) + ln * 4) = vc;
    if (p.k_held) *reinterpret_cast<bf16x8 *>(p.k_held + held) = from4x8(kc, scale4(ke));
    if (p.v_held) *reinterpret_cast<bf16x8 *>(p.v_held + held) = from4x8(vc, scale4(ve));
    // the row's scale bytes, K's and then V's: the blocks' quads hold one each
    constexpr int kBlocks = D / kBlock4;
    unsigned ks = ke << (8 * (ln / 4)), vs = ve << (8 * (ln / 4));
    #pragma unroll
    for (int off = 4; off < kLanes; off <<= 1) {
        ks |= __shfl_xor(ks, off);
        vs |= __shfl_xor(vs, off);
    }
    if (ln == 0) {
        if constexpr (kBlocks == 4)
            *reinterpret_cast<uint2 *>(p.scales + row * 8) = uint2{ks, vs};
        else
            *reinterpret_cast<unsigned *>(p.scales + row * 4) = ks | vs << 16;
    }
}

}  // namespace

hipError_t launch_kv4_write(const Kv4WriteParams &p, int B, int head_dim, hipStream_t s) {
    const int tokens = kWriteThreads / (head_dim / 8);
    const dim3 grid((unsigned)((p.T + tokens - 1) / tokens) * (unsigned)p.Hkv, (unsigned)B);
    return launch_kernel(head_dim == 64 ? kv4_write_kernel<64> : kv4_write_kernel<128>, grid, dim3(kWriteThreads), s, p);
}

}  // namespace tv
