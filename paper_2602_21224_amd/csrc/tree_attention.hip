// Tree-masked attention over a paged KV prefix for gfx950 (MI355X).
//
// What is computed (the paper's tree-shaped verification attention, §2.1, with
// the tree mask of SpecInfer cited in §8, over the paged cache of §7.1): for
// every sequence b, KV head g and query row (node i, query head h of g's
// group), the softmax-weighted sum of values over the whole committed prefix
// plus node i's own root path.
//
// Work decomposition
//   * A "row block" is up to 256 query rows of one (b, g): row r is node r / G,
//     head g * G + r % G, so the G heads sharing a KV head are batched and every
//     K/V tile is read once for all of them (GQA grouping).
//   * A "unit" is one (b, g, row block). Its work is a list of 64-key tiles: the
//     prefix tiles, then the tree tiles (tree nodes 0 .. the block's last node).
//     All units' tiles are laid end to end and the workgroups take equal
//     contiguous shares, so ragged prefixes stay balanced. A workgroup that
//     covers a whole unit writes the output directly; a split unit leaves
//     per-piece partials (max and sum in fp32, the piece's own normalised
//     output in bf16) that a second kernel merges with the usual log-sum-exp
//     rescaling.
//   * K and V tiles stream from HBM straight into a 4-stage LDS ring with
//     global_load_lds_dwordx4 (no register staging). Each 256-byte row is
//     stored with its 16-byte chunks XOR-swizzled by the key index, so the
//     MFMA operand reads below are free of bank conflicts. Keys past the
//     prefix, and tree slots past N, load a row that exists, of V tree node 0's
//     (finite), and are masked; the NaN-filled tail slots of a cache page are
//     never read.
//   * Each wave owns 32 query rows; the workgroup's 8 waves step through the
//     tiles together, one workgroup barrier per 64-key tile ("period"). In
//     period j every wave computes S^T = K_j Q^T with
//     v_mfma_f32_32x32x16_bf16 (keys on M, rows on N: a lane holds 16 scores
//     of one row, so a row max/sum needs one cross-half exchange) and
//     O^T += V_{j-1}^T P_{j-1}^T with the same instruction, and puts the
//     softmax work (mask, max, fp32 exponentials in base 2 with the scale
//     folded into one FMA, bf16 P^T) between those MFMAs, so that one wave's
//     matrix and vector work overlap. V^T operands come from the row-major
//     tile through ds_read_b64_tr_b16, which transposes 4x16 blocks on the
//     way out of LDS.
//   * At the end of period j each wave issues its share of K_{j+3} and
//     V_{j+2} in one burst: DMA writes into LDS slow down every wave's operand
//     reads, and a single burst per period disturbs them least. Each load is
//     issued about three periods before it is read.
//   * Reads of the ring are inline assembly with explicit lgkmcnt waits tied to
//     the fragments they produce, and ring hand-off is s_waitcnt vmcnt(n) +
//     s_barrier, so the compiler never inserts a blanket wait for the
//     in-flight tile loads.
//   * Tree visibility is a per-node ancestor bit set (256 bits) in LDS, built
//     by one wave while the first tiles load: for trees of up to 64 nodes each
//     lane follows its node's parent links through cross-lane shuffles, larger
//     trees use pointer doubling in LDS. A masked score is replaced by -inf
//     (selected, never added).
#include "tree_attention_kernel.h"

namespace tv {
namespace {

// Units taken whole have instances of their own, so that the split ones keep their
// code: with the choice inside the kernel it came out up to 0.8 % slower (45 nodes of
// head size 64 over 300-2500 keys 21.1 -> 21.3 us).
template <int D, int NW, bool NARROW>
hipError_t launch_main(const AttnParams &p, bool fine, hipStream_t s) {
    auto go = [&](auto kernel) { return launch_kernel(kernel, dim3(p.num_wg), dim3(NW * kWave), s, p); };
    if (fine && !p.whole_units)
        return p.small_pages ? go(tree_attention_kernel<D, NW, true, NARROW, false, true>)
                             : go(tree_attention_kernel<D, NW, false, NARROW, false, true>);
    if (p.whole_units)
        return p.small_pages ? go(tree_attention_kernel<D, NW, true, NARROW, true>)
                             : go(tree_attention_kernel<D, NW, false, NARROW, true>);
    return p.small_pages ? go(tree_attention_kernel<D, NW, true, NARROW, false>)
                         : go(tree_attention_kernel<D, NW, false, NARROW, false>);
}

template <int D, int NW>
hipError_t launch_dn(const AttnParams &p, bool fine, hipStream_t s) {
    hipError_t e;
    if constexpr (NW == 4)
        e = p.narrow ? launch_main<D, NW, true>(p, fine, s) : launch_main<D, NW, false>(p, fine, s);
    else
        e = launch_main<D, NW, false>(p, fine, s);
    if (e != hipSuccess) return e;
    if (p.num_wg > 1 && !p.whole_units) {
        constexpr int kRowsPerWg = 256 / (D / 8);
        const int chunks = (p.rows_per_block + kRowsPerWg - 1) / kRowsPerWg;
        const int stride = (p.num_wg + kNumXcd - 1) / kNumXcd * kNumXcd;
        e = launch_kernel(fine ? tree_attention_merge_fine_kernel<D> : tree_attention_merge_kernel<D>,
                          dim3(stride * chunks), dim3(256), s, p, stride);
    }
    return e;
}

template <int D>
hipError_t launch_d(const AttnParams &p, int waves, bool fine, hipStream_t s) {
    switch (waves) {
        case 4: return launch_dn<D, 4>(p, fine, s);
        case 8: return launch_dn<D, 8>(p, fine, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_tree_attention(const AttnParams &p, int head_dim, int waves, bool fine, hipStream_t s) {
    if (head_dim == 64) return launch_d<64>(p, waves, fine, s);
    if (head_dim == 128) return launch_d<128>(p, waves, fine, s);
    return hipErrorInvalidValue;
}

}  // namespace tv
