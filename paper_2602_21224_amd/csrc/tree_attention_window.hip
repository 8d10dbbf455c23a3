// Tree-masked attention inside a sliding window over a bf16 cache, for gfx950: the kernels
// of tree_attention.hip with a unit's prefix tiles cut to those that hold a visible key.
//
// Node i stands at position L + depth(i) and sees, of the prefix and of its root path, the
// positions t > L + depth(i) - window and t < sinks. The prefix tiles are the sinks' and
// those from the root's first visible position on, so the work is that of a prefix of about
// window + sinks tokens whatever L; only tiles at an edge are masked, per row, by the row's
// depth. Keys that no node sees are not read into a product, so their pages may be given
// back and their slots hold anything. Pieces of split units are kept in fp16 times a power
// of two per row, as in tree_verify_attention_shared.
//
// Measured: 32 sequences of 4096-32768 tokens, one node, a window of 4096 (8 KV heads of 128, 4
// query heads each) 118 us, 539 MB read at 4.6 TB/s, a copy's rate; 16 x 64 nodes, a window of 2048
// 65 us, of which 9-11 join split rows: the period of tree_verify_attention's tiles, 527
// TFLOP/s. Without a window, beside tree_verify_attention on the same batches: 16 sequences x 64
// nodes over 1024-4096 tokens 68.3 and 71.4, 4 x 256 over 16000 278 and 282, 32 x 1 over 1024-8192
// 121 and 125, 16 x 12 of 32 KV heads 86.2 and 82.7, one sequence x 64 over 2048 22.0 and 19.1.
#include "tree_attention_kernel.h"

namespace tv {
namespace {

template <int D, int NW, bool NARROW>
hipError_t launch_main(const WindowAttnParams &p, hipStream_t s) {
    auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(p.num_wg), dim3(NW * kWave), s, p); };
    if (p.whole_units)
        return p.small_pages ? go(tree_attention_kernel<D, NW, true, NARROW, true, false, true>)
                             : go(tree_attention_kernel<D, NW, false, NARROW, true, false, true>);
    return p.small_pages ? go(tree_attention_kernel<D, NW, true, NARROW, false, true, true>)
                         : go(tree_attention_kernel<D, NW, false, NARROW, false, true, true>);
}

template <int D>
hipError_t launch_d(const WindowAttnParams &p, int waves, hipStream_t s) {
    const hipError_t e = waves == 8  ? launch_main<D, 8, false>(p, s)
                         : p.narrow ? launch_main<D, 4, true>(p, s)
                                    : launch_main<D, 4, false>(p, s);
    if (e != hipSuccess || p.num_wg == 1 || p.whole_units) return e;
    constexpr int kRowsPerWg = 256 / (D / 8);
    const int chunks = (p.rows_per_block + kRowsPerWg - 1) / kRowsPerWg;
    const int stride = (p.num_wg + kNumXcd - 1) / kNumXcd * kNumXcd;
    return launch_kernel(tree_attention_merge_fine_kernel<D>, dim3(stride * chunks), dim3(256), s,
                         static_cast<const AttnParams &>(p), stride);
}

}  // namespace

hipError_t launch_window_attention(const WindowAttnParams &p, int head_dim, int waves, hipStream_t s) {
    if (head_dim == 64) return launch_d<64>(p, waves, s);
    if (head_dim == 128) return launch_d<128>(p, waves, s);
    return hipErrorInvalidValue;
}

}  // namespace tv
