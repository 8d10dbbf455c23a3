// C-ABI entry points of libtreeverify: argument checks, launch shapes and
// workspace carving. Every check runs on the host before any launch, so an
// error return means nothing was enqueued.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#define TREEVERIFY_BUILD 1
#include "treeverify.h"
#include "tv_internal.h"

namespace {

constexpr int kMaxDevices = 64;
constexpr int kWgPerCu = 1;          // the attention kernel's LDS ring allows one workgroup per CU
constexpr int kMinShareTiles = 2;    // smallest per-workgroup share (measured: 8 -> 2 is -26 % at 8B bs1)
constexpr int kSetupTiles = 3;       // measured cost of starting a unit piece, in 64-key tiles
constexpr int kArgmaxMinWorkgroups = 2048;
constexpr int kArgmaxMinSegment = 4096;

int g_cu_count[kMaxDevices];         // 0 = not yet queried
int g_is_gfx950[kMaxDevices];        // 0 = not yet queried, 1 = yes, -1 = no

// Scratch of tree_argmax_accept_noalloc: one copy per GPU, held until the
// process ends. Host code never names it directly (its host-side name is a
// stand-in, not a device address); it uses the per-device address that
// hipGetSymbolAddress returns, looked up once per device on the first call.
static __device__ __align__(256) unsigned char scratch[TV_NOALLOC_SCRATCH_BYTES];
std::atomic<void *> g_scratch_ptr[kMaxDevices];

// Device address of the current device's scratch, or nullptr if the lookup fails.
void *scratch_ptr() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    void *ptr = g_scratch_ptr[dev].load(std::memory_order_acquire);
    if (ptr == nullptr) {
        // Two threads may race here; both store the same address.
        if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)) != hipSuccess || ptr == nullptr)
            return nullptr;
        g_scratch_ptr[dev].store(ptr, std::memory_order_release);
    }
    return ptr;
}

bool device_ok() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return false;
    if (g_is_gfx950[dev] == 0) {
        hipDeviceProp_t prop;
        const bool ok = hipGetDeviceProperties(&prop, dev) == hipSuccess &&
                        strncmp(prop.gcnArchName, "gfx950", 6) == 0;
        g_is_gfx950[dev] = ok ? 1 : -1;
    }
    return g_is_gfx950[dev] == 1;
}

int cu_count() {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
    if (g_cu_count[dev] == 0) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0)
            n = 256;
        g_cu_count[dev] = n;
    }
    return g_cu_count[dev];
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// Whether two int32 arrays of n elements share any.
bool overlap(const int32_t *a, const int32_t *b, long n) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return (x < y ? y - x : x - y) < (uintptr_t)n * sizeof(int32_t);
}
bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

struct AttnShape {
    int G, rows, waves, rows_per_block, row_blocks, tree_tiles_all;
};

AttnShape attn_shape(int N, int Hq, int Hkv) {
    AttnShape s;
    s.G = Hq / Hkv;
    s.rows = N * s.G;
    // Four waves at least: a workgroup of fewer waves leaves a unit's tile
    // loads to one or two waves (and the one-wave kernel spills), which
    // measured 11x (one wave) and 1.2x (two waves) slower on 12-row units
    // than four waves with the extra rows idle.
    const int need = (s.rows + tv::kRowsPerWave - 1) / tv::kRowsPerWave;
    s.waves = need > 4 ? 8 : 4;
    s.rows_per_block = s.waves * tv::kRowsPerWave;
    s.row_blocks = (s.rows + s.rows_per_block - 1) / s.rows_per_block;
    s.tree_tiles_all = 0;
    for (int rb = 0; rb < s.row_blocks; ++rb) {
        const int last_row = (rb + 1) * s.rows_per_block < s.rows ? (rb + 1) * s.rows_per_block - 1
                                                                  : s.rows - 1;
        const int jmax = last_row / s.G + 1;
        s.tree_tiles_all += (jmax + tv::kKeyTile - 1) / tv::kKeyTile;
    }
    return s;
}

struct AttnWorkspace {
    size_t o_bytes, ml_bytes, desc_bytes, total;
};

AttnWorkspace attn_workspace(const AttnShape &s, int D, int max_wg, bool fine = false) {
    AttnWorkspace w;
    w.o_bytes = round_up((size_t)max_wg * 2 * s.rows_per_block * D * sizeof(uint16_t), 256);
    w.ml_bytes = round_up((size_t)max_wg * 2 * s.rows_per_block * (fine ? 4 : 2) * sizeof(float), 256);
    w.desc_bytes = round_up((size_t)max_wg * 4 * sizeof(int32_t), 256);
    w.total = w.o_bytes + w.ml_bytes + w.desc_bytes;
    return w;
}

// Batches with shared prefixes run workgroups of eight waves throughout: a
// group's rows are many. Own units of at most kOwnRows rows are taken wave by wave
// (tree_attention_own.h), larger ones in row blocks like the shared ones: 16 sequences
// with 32, 48 and 64 rows over 4096 shared and up to 1024 own tokens 37, 42 and 67 us
// wave by wave, 42, 46 and 50 in row blocks.
constexpr int kOwnRows = 48;

struct SharedShape {
    AttnShape wide;
    int own_rows, own_tiles16, own_blocks;
};

SharedShape shared_shape(int N, int Hq, int Hkv) {
    SharedShape s;
    s.wide = attn_shape(N, Hq, Hkv);
    s.wide.waves = 8;
    s.wide.rows_per_block = s.wide.waves * tv::kRowsPerWave;
    s.wide.row_blocks = (s.wide.rows + s.wide.rows_per_block - 1) / s.wide.rows_per_block;
    s.wide.tree_tiles_all = s.wide.row_blocks * ((N + tv::kKeyTile - 1) / tv::kKeyTile);   // at most
    s.own_tiles16 = s.wide.rows <= kOwnRows ? (s.wide.rows + 15) / 16 : 0;
    s.own_rows = s.own_tiles16 ? 16 * s.own_tiles16 : s.wide.rows_per_block;
    s.own_blocks = s.own_tiles16 ? 1 : s.wide.row_blocks;
    return s;
}

// Whether the keys are taken by groups at all. That has tables to build and every row's
// two parts to join, 5 to 10 us, so it has to save more: K/V rows that the plain launch
// reads again (which it often finds in the caches), or row blocks. us, plain and by groups:
// at most 19 MB of K/V rows saved 24.4 and 29.9 (3 sequences of 3 rows, two groups), 17 MB
// 19.6 and 28.5 (3 of 5 rows), 30 MB 23.2 and 25.7 (36 of 32, 12 groups), 34 MB 33.4 and 28.3
// (4 of 56, two groups), 39 MB 25.7 and 26.3 (4 of 4), 44 MB 26.9 and 18.8 (36 of 8, two
// groups), 63 MB 28.4 and 26.0 (11 of 7). And of the rows of a sequence's blocks of 256 a
// quarter has to be empty, which a group's rows fill: 208 rows 105 and 108, 232 rows 55 and
// 52, 427 rows 32.7 and 35.9, 775 rows 260 and 242, 1824 rows 467 and 569, 154 rows 62 and
// 46. Row blocks of eight waves also have to save more tiles than they cost, by the count
// that the kernel makes of each group: 29 sequences of 273 rows over 154 tokens 118 and 133.
bool sharing_pays(const AttnShape &s, int B, int Hkv, int D, int groups, long max_len) {
    if (groups == 0 || groups >= B) return false;            // one sequence per group (empty ones count)
    if ((long)(B - groups) * Hkv * D * 4 * max_len < 32l << 20) return false;
    const long block = 8 * tv::kRowsPerWave, padded = (s.rows + block - 1) / block * block;
    if ((padded - s.rows) * 4 < padded) return false;
    if (s.rows <= kOwnRows) return true;
    const long apart = B * (padded / block), together = (B * (long)s.rows + block - 1) / block;
    return (apart - together) * (max_len / tv::kKeyTile) > kSetupTiles * together + tv::kJoinTiles * apart;
}

// Most row blocks per KV head that the groups' shared units can have together.
long shared_blocks(const SharedShape &s, int B, int groups) {
    return ((long)B * s.wide.rows + s.wide.rows_per_block - 1) / s.wide.rows_per_block + groups;
}

struct SharedWorkspace {
    size_t o, piece, whole, row, unit, seq, own_o, own_piece, total;       // byte offsets, and the whole
};

SharedWorkspace shared_workspace(const SharedShape &s, int B, int N, int Hq, int Hkv, int D, int groups,
                                 int max_wg) {
    const size_t rows = (size_t)B * N * Hq;
    const size_t units = ((size_t)B * s.own_blocks + (size_t)shared_blocks(s, B, groups)) * Hkv;
    const size_t slots = (size_t)max_wg * 2 * s.wide.rows_per_block;                        // rows of them
    const size_t own = s.own_tiles16 ? (size_t)max_wg * s.wide.waves * 2 * s.own_rows : 0;   // of the waves'
    SharedWorkspace w;
    size_t at = 0;
    auto take = [&](size_t elements, size_t bytes) {
        const size_t from = at;
        at += round_up(elements * bytes, 256);
        return from;
    };
    w.o = take(slots * D, sizeof(uint16_t));
    w.piece = take(slots * 4, sizeof(float));
    w.whole = take(rows * 2 * D, sizeof(uint16_t));
    w.row = take(rows * 2 * 4, sizeof(float));
    w.unit = take(units * 2, sizeof(int32_t));
    w.seq = take((size_t)B * 4, sizeof(int32_t));
    w.own_o = take(own * D, sizeof(uint16_t));
    w.own_piece = take(own * 4, sizeof(float));
    w.total = at + 256;
    const size_t plain = attn_workspace(attn_shape(N, Hq, Hkv), D, max_wg, true).total;
    if (w.total < plain) w.total = plain;
    return w;
}

bool attn_shape_ok(int B, int N, int Hq, int Hkv, int D) {
    if (B < 0 || B > tv::kMaxBatchAttn) return false;
    if (N < 1 || N > tv::kMaxNodes) return false;
    if (D != 64 && D != 128) return false;
    if (Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return false;
    if ((long)(Hq / Hkv) * N > 2048) return false;
    // 256 key rows of all KV heads (a page, or the tree's rows) stay below 4 GiB,
    // so in-kernel row offsets fit 32 bits
    if ((long)Hkv * D * 2 * 256 >= (1l << 32)) return false;
    return true;
}

void argmax_plan(int B, int N, int V, int *segs, int *seg_len) {
    const long rows = (long)B * N;
    long s = rows > 0 ? (kArgmaxMinWorkgroups + rows - 1) / rows : 1;
    const long max_s = ((long)V + kArgmaxMinSegment - 1) / kArgmaxMinSegment;
    if (s > max_s) s = max_s;
    if (s < 1) s = 1;
    if (s > 65535) s = 65535;
    long len = ((long)V + s - 1) / s;
    len = (len + 3) / 4 * 4;
    s = ((long)V + len - 1) / len;
    *segs = (int)s;
    *seg_len = (int)len;
}

// Virtual tiles of a launch of tree_verify_attention over prefixes of `len` tokens. They
// are counted in int32 on the device: fewer than kMaxTiles for any kv_len.
constexpr long kMaxTiles = 1l << 30;

long attn_tiles(const AttnShape &s, int B, int Hkv, long len) {
    return (long)B * Hkv *
           ((long)s.row_blocks * ((len + tv::kKeyTile - 1) / tv::kKeyTile + kSetupTiles) + s.tree_tiles_all);
}

// The same of a launch that takes keys by groups; small own units count places (tree_attention_own.h).
long shared_places(const SharedShape &s, int B, int N, int Hkv, int D, int groups, long len) {
    const long prefix = (len + tv::kKeyTile - 1) / tv::kKeyTile + kSetupTiles, keys = tv::own_keys(D);
    const long own = s.own_tiles16 ? (len + N + keys - 1) / keys * tv::kOwnTile + 1
                                   : s.own_blocks * prefix + s.wide.tree_tiles_all;
    return Hkv * (shared_blocks(s, B, groups) * prefix + B * own);
}

// Whether each unit is taken whole by a workgroup of its own, over `tiles` prefix tiles at most.
// Short units are not worth splitting: one workgroup per unit saves the merge
// launch and the partials it reads, 3-4 us, for about 1.2 us per tile of a
// unit of at most 16 rows or of head size 64, and 2 us of the others. While the
// units leave CUs idle, long ones (several row blocks, or one-token pages of head
// size 128, each load a page) are split a tile sooner. Measured (us per call,
// whole and split): 16 rows of 64, 4 tiles 10.5 and 12.6; 16 rows of 128, 4 tiles
// 13.0 and 13.9, with one-token pages 64 units 14.4 and 13.8, 128 units 13.0 and
// 14.4; 132 rows of 128, 3 tiles 14.5 and 16.4; 256 rows of 128, 3 tiles 14.9 and
// 15.0, 4 tiles 16.9 and 15.0; 512 rows of 64, 4 tiles, 16 units 15.9 and 15.4;
// 1024 rows of 64, 4 tiles, 8 units 14.4 and 13.7; 2048 rows of 64, 4 tiles, 16
// units 18.8 and 17.3; 2048 rows of 128, 3 tiles, 16 units 20.0 and 18.8.
bool whole_units(const AttnShape &s, int B, int N, int Hkv, int D, long tiles, bool small_pages, int max_wg) {
    const long units = (long)B * Hkv * s.row_blocks;
    const long unit_tiles = tiles + (N + tv::kKeyTile - 1) / tv::kKeyTile;
    const bool sooner = D == 64          ? s.rows > 256 && units < 128
                        : s.rows <= 16 ? small_pages && units < 128
                                       : s.rows > 512 && units < 32;
    return units <= max_wg && unit_tiles <= (D == 64 || s.rows <= 16 ? 4 : 3) - (sooner ? 1 : 0);
}

// tree_verify_attention behind its argument checks; `fine`: see launch_tree_attention.
int launch_attention(bool fine, const uint16_t *q, const uint16_t *k_tree, const uint16_t *v_tree,
                     const uint16_t *k_cache, const uint16_t *v_cache, const int32_t *page_table, const int32_t *kv_len,
                     const int32_t *parent, const int32_t *num_nodes, int B, int N, int Hq, int Hkv, int D, int P,
                     int max_pages, int num_pages, int max_kv_len, float scale, uint16_t *out, float *lse,
                     void *workspace, size_t workspace_bytes, hipStream_t stream) {
    const AttnShape s = attn_shape(N, Hq, Hkv);
    const int max_wg = cu_count() * kWgPerCu;
    const AttnWorkspace ws = attn_workspace(s, D, max_wg, fine);
    if (workspace_bytes < ws.total) return TV_ERR_WORKSPACE;

    const long max_len = (long)max_pages * P;
    if (attn_tiles(s, B, Hkv, max_len) >= kMaxTiles) return TV_ERR_SHAPE;

    const long hint_len = max_kv_len < max_len ? max_kv_len : max_len;
    long num_wg = attn_tiles(s, B, Hkv, hint_len) / kMinShareTiles;
    if (num_wg < 1) num_wg = 1;
    if (num_wg > max_wg) num_wg = max_wg;
    const bool small_pages = P < 1024 / (2 * D);
    const bool whole =
        whole_units(s, B, N, Hkv, D, (hint_len + tv::kKeyTile - 1) / tv::kKeyTile, small_pages, max_wg);
    if (whole) num_wg = (long)B * Hkv * s.row_blocks;

    tv::AttnParams p;
    p.q = q; p.k_tree = k_tree; p.v_tree = v_tree; p.k_cache = k_cache; p.v_cache = v_cache;
    p.page_table = page_table; p.kv_len = kv_len; p.parent = parent; p.num_nodes = num_nodes;
    p.out = out; p.lse = lse;
    char *base = static_cast<char *>(workspace);
    p.ws_o = reinterpret_cast<uint16_t *>(base);
    p.ws_ml = reinterpret_cast<float *>(base + ws.o_bytes);
    p.ws_desc = reinterpret_cast<int32_t *>(base + ws.o_bytes + ws.ml_bytes);
    p.B = B; p.N = N; p.Hq = Hq; p.Hkv = Hkv; p.G = s.G;
    p.P = P; p.p_shift = __builtin_ctz((unsigned)P);
    p.max_pages = max_pages; p.num_pages = num_pages;
    p.rows_per_block = s.rows_per_block;
    p.setup_tiles = kSetupTiles;
    p.small_pages = small_pages ? 1 : 0;
    p.narrow = s.rows <= 16 ? 1 : 0;
    p.num_wg = (int)num_wg;
    p.whole_units = whole ? 1 : 0;
    const float sc = scale > 0.f ? scale : 1.0f / sqrtf((float)D);
    p.scale = sc;
    p.scale_log2 = sc * 1.4426950408889634f;

    return tv::launch_tree_attention(p, D, s.waves, fine, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

// What the calls with a window have in common: limits of sizes, prefix tiles of a unit, and
// the parameters that do not depend on the kernel.
bool window_shape_ok(int B, int N, int Hq, int Hkv, int D, int P, int max_pages, int num_pages, int max_kv_len,
                     int window, int sinks) {
    return attn_shape_ok(B, N, Hq, Hkv, D) && pow2(P) && P <= 256 && max_pages >= 1 && num_pages >= 1 &&
           max_kv_len >= 0 && window >= 0 && sinks >= 0 &&
           (long)max_pages * P <= tv::kMaxPrefix;
}

long window_tiles(long len, int window, int sinks) {
    const long all = (len + tv::kKeyTile - 1) / tv::kKeyTile;
    if (window == 0) return all;
    const long some = ((long)window + tv::kKeyTile - 2) / tv::kKeyTile + 1 + ((long)sinks + tv::kKeyTile - 1) / tv::kKeyTile;
    return all < some ? all : some;
}

void window_params(tv::WindowAttnParams &p, const uint16_t *q, const uint16_t *k_tree, const uint16_t *v_tree,
                   const int32_t *page_table, const int32_t *kv_len, const int32_t *parent, const int32_t *num_nodes,
                   int B, int N, int Hq, int Hkv, int D, int P, int max_pages, int num_pages, int window, int sinks,
                   float scale, uint16_t *out, float *lse, void *workspace, const AttnWorkspace &ws) {
    p.q = q; p.k_tree = k_tree; p.v_tree = v_tree;
    p.page_table = page_table; p.kv_len = kv_len; p.parent = parent; p.num_nodes = num_nodes;
    p.out = out; p.lse = lse;
    char *base = static_cast<char *>(workspace);
    p.ws_o = reinterpret_cast<uint16_t *>(base);
    p.ws_ml = reinterpret_cast<float *>(base + ws.o_bytes);
    p.ws_desc = reinterpret_cast<int32_t *>(base + ws.o_bytes + ws.ml_bytes);
    p.B = B; p.N = N; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv;
    p.P = P; p.p_shift = __builtin_ctz((unsigned)P);
    p.max_pages = max_pages; p.num_pages = num_pages;
    p.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)D);
    p.scale_log2 = p.scale * 1.4426950408889634f;
    p.window = window; p.sinks = sinks;
}

// Attention over a cache in 4 bits: few rows per KV head wave by wave, in blocks of 16 or 32
// rows (tree_attention_kv4.hip), many in blocks of 128 or 256 by workgroups
// (tree_attention_kv4_wide.hip). Measured (us per call, head size 128, by waves and by
// workgroups): 64 sequences of 200-500 tokens, 64 rows 50 and 56, 68 rows 62 and 56, 96 rows 67
// and 57 (every block takes the tree's tiles again); 16 sequences of 500-900 tokens, 96 rows 35
// and 32; of 1024-4096 tokens, 64 rows 41 and 62, 96 rows 51 and 63, 128 rows 63 and 64, 160 rows
// 73 and 67; 4 sequences of 32768 tokens, 128 rows 115 and 154, 160 rows 142 and 165, 192 rows
// 162 and 166. Head size 64 has its line in nearly the same place: 64 sequences of 200-500 tokens,
// 64 rows 35 and 42, 68 rows 43 and 42; 16 of 500-900, 64 rows 21.1 and 23.4, 96 rows 24.1 both; of
// 1024-4096, 96 rows 36 and 45, 128 rows 44 and 46, 160 rows 51 both; 4 of 32768, 160 rows 95 and
// 117, 192 rows 110 and 118 (the line costs it 4 and 7 % at 128 and 192 rows).
// Shares: of 2, 4, 6, 8 and 12 set-up tiles per unit and 4, 6 and 8 tiles at least per share the
// smallest calls took 17.3 to 13.3, 8 and 8 13.8, the larger ones the same within their noise.
constexpr int kv4_stream_rows(long prefix) {
    return prefix < 1024 ? 64 : prefix < 16384 ? 96 : 160;
}
constexpr int kKv4StreamSetupTiles = 8;
constexpr int kKv4StreamMinShareTiles = 8;
constexpr int kKv4StreamWgPerCu = 2;

struct Kv4Shape : AttnShape {
    bool stream;
    int max_wg, setup;
};

Kv4Shape kv4_shape(int N, int Hq, int Hkv, bool stream) {
    Kv4Shape s;
    static_cast<AttnShape &>(s) = attn_shape(N, Hq, Hkv);
    s.stream = stream;
    s.setup = stream ? kKv4StreamSetupTiles : kSetupTiles;
    s.max_wg = cu_count() * (s.stream ? kKv4StreamWgPerCu : kWgPerCu);
    s.rows_per_block = s.stream ? (s.rows <= 16 ? 16 : 32) : s.rows <= 128 ? 128 : 256;
    s.row_blocks = (s.rows + s.rows_per_block - 1) / s.rows_per_block;
    s.tree_tiles_all = s.row_blocks * ((N + tv::kKeyTile - 1) / tv::kKeyTile);      // at most
    return s;
}

// Virtual tiles of such a launch over `tiles` prefix tiles.
long kv4_tiles(const Kv4Shape &s, int B, int Hkv, long tiles) {
    return (long)B * Hkv * ((long)s.row_blocks * (tiles + s.setup) + s.tree_tiles_all);
}

}  // namespace

extern "C" {

int tv_abi_version(void) { return TV_ABI_VERSION; }

const char *tv_status_string(int status) {
    switch (status) {
        case TV_OK: return "ok";
        case TV_ERR_NULL: return "a required pointer is NULL";
        case TV_ERR_SHAPE: return "a size or count is outside the supported range";
        case TV_ERR_ALIGN: return "a tensor pointer is not 16-byte aligned";
        case TV_ERR_WORKSPACE: return "workspace missing or smaller than required";
        case TV_ERR_HIP: return "a HIP runtime call or kernel launch failed";
        case TV_ERR_DEVICE: return "the current device is not gfx950";
        case TV_ERR_SCRATCH:
            return "the call needs more scratch than the library's static buffer holds "
                   "(TV_NOALLOC_SCRATCH_BYTES)";
        case TV_ERR_OVERLAP: return "an output array overlaps an input that it may not overlap";
        default: return "unknown status";
    }
}

size_t tv_attention_workspace_size(int B, int N, int Hq, int Hkv, int D) {
    if (!attn_shape_ok(B, N, Hq, Hkv, D)) return 0;
    const AttnShape s = attn_shape(N, Hq, Hkv);
    return attn_workspace(s, D, cu_count() * kWgPerCu).total;
}

int tree_verify_attention(const uint16_t *q, const uint16_t *k_tree, const uint16_t *v_tree,
                          const uint16_t *k_cache, const uint16_t *v_cache,
                          const int32_t *page_table, const int32_t *kv_len, const int32_t *parent,
                          const int32_t *num_nodes, int B, int N, int Hq, int Hkv, int D, int P,
                          int max_pages, int num_pages, int max_kv_len, float scale, uint16_t *out,
                          float *lse,
                          void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!attn_shape_ok(B, N, Hq, Hkv, D)) return TV_ERR_SHAPE;
    if (!pow2(P) || P > 256 || max_pages < 1 || num_pages < 1 || max_kv_len < 0)
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!q || !k_tree || !v_tree || !k_cache || !v_cache || !page_table || !kv_len || !parent ||
        !out || !workspace)
        return TV_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(k_cache) ||
        !aligned16(v_cache) || !aligned16(out) || !aligned16(workspace))
        return TV_ERR_ALIGN;
    if (!device_ok()) return TV_ERR_DEVICE;

    return launch_attention(false, q, k_tree, v_tree, k_cache, v_cache, page_table, kv_len, parent, num_nodes, B,
                            N, Hq, Hkv, D, P, max_pages, num_pages, max_kv_len, scale, out, lse, workspace,
                            workspace_bytes, stream);
}

size_t tv_argmax_workspace_size(int B, int N, int V) {
    if (B < 0 || B > 65535 || N < 1 || N > tv::kMaxNodes || V < 1) return 0;
    int segs = 1, seg_len = 4;
    argmax_plan(B, N, V, &segs, &seg_len);
    return round_up((size_t)B * N * segs * sizeof(unsigned long long), 256) + 256;
}

}  // extern "C"

namespace {

// Argument checks and launches shared by tree_argmax_accept and its no-alloc
// variant; `ws` is the per-(row, segment) key buffer (every slot the accept
// kernel reads is written earlier in the same call).
int argmax_accept_checked(const float *logits, const int32_t *draft_tokens, const int32_t *parent,
                          const int32_t *num_nodes, int B, int N, int V, int32_t *argmax_out,
                          int32_t *accept_len, int32_t *accept_idx, int32_t *bonus_token,
                          void *ws, hipStream_t stream) {
    int segs = 1, seg_len = 4;
    argmax_plan(B, N, V, &segs, &seg_len);
    const hipError_t e = tv::launch_argmax_accept(
        logits, draft_tokens, parent, num_nodes, B, N, V, segs, seg_len, argmax_out, accept_len,
        accept_idx, bonus_token, static_cast<unsigned long long *>(ws), stream);
    return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

bool argmax_args_ok(int B, int N, int V) {
    return B >= 0 && B <= 65535 && N >= 1 && N <= tv::kMaxNodes && V >= 1;
}

bool argmax_ptrs_ok(const float *logits, const int32_t *draft_tokens, const int32_t *parent,
                    int32_t *argmax_out, int32_t *accept_len, int32_t *accept_idx,
                    int32_t *bonus_token) {
    return logits && draft_tokens && parent && argmax_out && accept_len && accept_idx &&
           bonus_token;
}

}  // namespace

extern "C" {

int tree_argmax_accept(const float *logits, const int32_t *draft_tokens, const int32_t *parent,
                       const int32_t *num_nodes, int B, int N, int V, int32_t *argmax_out,
                       int32_t *accept_len,
                       int32_t *accept_idx, int32_t *bonus_token, void *workspace,
                       size_t workspace_bytes, hipStream_t stream) {
    if (!argmax_args_ok(B, N, V)) return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!argmax_ptrs_ok(logits, draft_tokens, parent, argmax_out, accept_len, accept_idx,
                        bonus_token) || !workspace)
        return TV_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(logits) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 7u))
        return TV_ERR_ALIGN;
    if (workspace_bytes < tv_argmax_workspace_size(B, N, V)) return TV_ERR_WORKSPACE;
    if (!device_ok()) return TV_ERR_DEVICE;
    return argmax_accept_checked(logits, draft_tokens, parent, num_nodes, B, N, V, argmax_out,
                                 accept_len, accept_idx, bonus_token, workspace, stream);
}

int tree_argmax_accept_noalloc(const float *logits, const int32_t *draft_tokens,
                               const int32_t *parent, const int32_t *num_nodes, int B, int N,
                               int V, int32_t *argmax_out, int32_t *accept_len,
                               int32_t *accept_idx, int32_t *bonus_token, hipStream_t stream) {
    if (!argmax_args_ok(B, N, V)) return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!argmax_ptrs_ok(logits, draft_tokens, parent, argmax_out, accept_len, accept_idx,
                        bonus_token))
        return TV_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(logits) & 3u) return TV_ERR_ALIGN;
    if (tv_argmax_workspace_size(B, N, V) > (size_t)TV_NOALLOC_SCRATCH_BYTES)
        return TV_ERR_SCRATCH;
    if (!device_ok()) return TV_ERR_DEVICE;
    void *ws = scratch_ptr();
    if (ws == nullptr) return TV_ERR_HIP;
    return argmax_accept_checked(logits, draft_tokens, parent, num_nodes, B, N, V, argmax_out,
                                 accept_len, accept_idx, bonus_token, ws, stream);
}

int kv_compact_accepted(const uint16_t *k_tree, const uint16_t *v_tree, uint16_t *k_cache,
                        uint16_t *v_cache, const int32_t *page_table, const int32_t *kv_len,
                        const int32_t *accept_idx, const int32_t *accept_len, int B, int N,
                        int Hkv, int D, int P, int max_pages, int num_pages, hipStream_t stream) {
    if (B < 0 || B > 65535 || N < 1 || N > tv::kMaxNodes || Hkv < 1 || D < 1 ||
        ((long)Hkv * D) % 8 != 0 || !pow2(P) || P > 256 || max_pages < 1 || num_pages < 1)
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!k_tree || !v_tree || !k_cache || !v_cache || !page_table || !kv_len || !accept_idx ||
        !accept_len)
        return TV_ERR_NULL;
    if (!aligned16(k_tree) || !aligned16(v_tree) || !aligned16(k_cache) || !aligned16(v_cache))
        return TV_ERR_ALIGN;
    if (!device_ok()) return TV_ERR_DEVICE;
    const hipError_t e = tv::launch_kv_compact(k_tree, v_tree, k_cache, v_cache, page_table,
                                               kv_len, accept_idx, accept_len, B, N, Hkv, D, P,
                                               max_pages, num_pages, stream);
    return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

static bool shared_shape_ok(int B, int N, int Hq, int Hkv, int D, int groups) {
    return attn_shape_ok(B, N, Hq, Hkv, D) && B <= tv::kMaxBatchShared && groups >= 0 &&
           groups <= tv::kMaxGroups &&
           (long)B * N * Hq * D <= (1l << 34);          // the joining kernel's threads, 8 values each
}

size_t tv_shared_attention_workspace_size(int B, int N, int Hq, int Hkv, int D, int groups) {
    if (!shared_shape_ok(B, N, Hq, Hkv, D, groups)) return 0;
    return shared_workspace(shared_shape(N, Hq, Hkv), B, N, Hq, Hkv, D, groups, cu_count() * kWgPerCu).total;
}

int tree_verify_attention_shared(
    const uint16_t *q, const uint16_t *k_tree, const uint16_t *v_tree, const uint16_t *k_cache,
    const uint16_t *v_cache, const int32_t *page_table, const int32_t *kv_len,
    const int32_t *parent, const int32_t *num_nodes, const int32_t *group_start,
    const int32_t *shared_len, int groups, int B, int N, int Hq, int Hkv, int D, int P,
    int max_pages, int num_pages, int max_kv_len, float scale, uint16_t *out, float *lse,
    void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!shared_shape_ok(B, N, Hq, Hkv, D, groups)) return TV_ERR_SHAPE;
    if (!pow2(P) || P > 256 || max_pages < 1 || num_pages < 1 || max_kv_len < 0 ||
        (long)max_pages * P > INT32_MAX)
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!q || !k_tree || !v_tree || !k_cache || !v_cache || !page_table || !kv_len || !parent ||
        !out || !workspace || (groups > 0 && (!group_start || !shared_len)))
        return TV_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(k_cache) ||
        !aligned16(v_cache) || !aligned16(out) || !aligned16(workspace))
        return TV_ERR_ALIGN;
    const SharedShape s = shared_shape(N, Hq, Hkv);
    const int max_wg = cu_count() * kWgPerCu;
    const SharedWorkspace ws = shared_workspace(s, B, N, Hq, Hkv, D, groups, max_wg);
    if (workspace_bytes < ws.total) return TV_ERR_WORKSPACE;
    // Tables that hold longer prefixes than keys taken by groups can be counted for take the
    // plain launch, too: what it accepts is accepted.
    const long max_len = (long)max_pages * P, hint_len = max_kv_len < max_len ? max_kv_len : max_len;
    const bool grouped = shared_places(s, B, N, Hkv, D, groups, max_len) < kMaxTiles &&
                         sharing_pays(s.wide, B, Hkv, D, groups, hint_len);
    if (!grouped && attn_tiles(attn_shape(N, Hq, Hkv), B, Hkv, max_len) >= kMaxTiles) return TV_ERR_SHAPE;
    if (!device_ok()) return TV_ERR_DEVICE;
    if (!grouped)
        return launch_attention(true, q, k_tree, v_tree, k_cache, v_cache, page_table, kv_len, parent, num_nodes,
                                B, N, Hq, Hkv, D, P, max_pages, num_pages, max_kv_len, scale, out, lse, workspace,
                                workspace_bytes, stream);
    const long blocks = (long)B * s.own_blocks + shared_blocks(s, B, groups);
    long num_wg = Hkv * (blocks * ((hint_len + tv::kKeyTile - 1) / tv::kKeyTile + kSetupTiles) +
                         (long)B * s.wide.tree_tiles_all) / kMinShareTiles;
    if (num_wg < 1) num_wg = 1;
    if (num_wg > max_wg) num_wg = max_wg;
    // the two kinds of units divide the workgroups in multiples of the XCDs, both at least one
    if (s.own_tiles16) num_wg = num_wg < 2 * tv::kNumXcd ? 2 * tv::kNumXcd : num_wg / tv::kNumXcd * tv::kNumXcd;

    tv::SharedAttnParams p{};
    p.q = q; p.k_tree = k_tree; p.v_tree = v_tree; p.k_cache = k_cache; p.v_cache = v_cache;
    p.page_table = page_table; p.kv_len = kv_len; p.parent = parent; p.num_nodes = num_nodes;
    p.out = out; p.lse = lse;
    p.B = B; p.N = N; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv;
    p.P = P; p.p_shift = __builtin_ctz((unsigned)P);
    p.max_pages = max_pages; p.num_pages = num_pages;
    p.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)D);
    p.scale_log2 = p.scale * 1.4426950408889634f;
    char *base = static_cast<char *>(workspace);
    auto halves = [&](size_t off) { return reinterpret_cast<uint16_t *>(base + off); };
    auto ints = [&](size_t off) { return reinterpret_cast<int32_t *>(base + off); };
    auto quads = [&](size_t off) { return reinterpret_cast<tv::f32x4 *>(base + off); };
    p.ws_o = halves(ws.o);
    p.ws_piece = quads(ws.piece);
    p.ws_whole = halves(ws.whole);
    p.ws_row = quads(ws.row);
    p.ws_unit = ints(ws.unit);
    p.ws_seq = ints(ws.seq);
    p.own_rows = s.own_rows; p.own_tiles16 = s.own_tiles16;
    p.own_o = s.own_tiles16 ? halves(ws.own_o) : p.ws_o;
    p.own_piece = s.own_tiles16 ? quads(ws.own_piece) : p.ws_piece;
    p.group_start = group_start; p.shared_len = shared_len; p.groups = groups;
    p.rows_per_block = s.wide.rows_per_block;
    p.setup_tiles = kSetupTiles;
    p.small_pages = P < 1024 / (2 * D) ? 1 : 0;
    p.num_wg = (int)num_wg;
    return tv::launch_shared_attention(p, D, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

int kv_accumulate_weights(const uint16_t *q, const float *lse, const uint16_t *k_cache,
                          const int32_t *page_table, const int32_t *kv_len,
                          const int32_t *accept_idx, const int32_t *accept_len,
                          const int32_t *seen, const int32_t *fixed_len, const float *weight,
                          int B, int N, int Hq, int Hkv, int D, int P, int max_pages,
                          int num_pages, int max_kv_len, float scale, float *weight_out,
                          int32_t *position, hipStream_t stream) {
    if (B < 0 || B > 65535 || Hkv > 65535 || !attn_shape_ok(1, N, Hq, Hkv, D) || !pow2(P) ||
        P > 256 || max_pages < 1 || num_pages < 1 || max_kv_len < 0 ||
        (long)max_pages * P > (1l << 24))
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!q || !lse || !k_cache || !page_table || !kv_len || !accept_idx || !accept_len || !seen ||
        !weight || !weight_out || !position)
        return TV_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_cache)) return TV_ERR_ALIGN;
    if (!device_ok()) return TV_ERR_DEVICE;
    tv::WeightParams p;
    p.q = q; p.k_cache = k_cache; p.lse = lse; p.weight = weight;
    p.page_table = page_table; p.kv_len = kv_len; p.accept_idx = accept_idx;
    p.accept_len = accept_len; p.seen = seen; p.fixed_len = fixed_len;
    p.weight_out = weight_out; p.position = position;
    p.B = B; p.N = N; p.Hq = Hq; p.Hkv = Hkv;
    p.p_shift = __builtin_ctz((unsigned)P); p.max_pages = max_pages; p.num_pages = num_pages;
    p.g_inv = Hq == Hkv ? 0u : (unsigned)((1ull << 32) / (unsigned)(Hq / Hkv) + 1);
    const long cap = (long)max_pages * P, hint = (long)max_kv_len + N;
    p.max_keys = (int)(hint < cap ? hint : cap);
    p.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)D);
    return tv::launch_accumulate_weights(p, D, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

static bool evict_shape_ok(int B, int Hkv, int max_pages, int P) {
    return B >= 0 && B <= 65535 && Hkv >= 1 && Hkv <= 65535 && max_pages >= 1 && pow2(P) &&
           P <= 256 && (long)max_pages * P <= (1l << 24);
}

size_t tv_evict_workspace_size(int B, int Hkv, int max_pages, int P) {
    if (!evict_shape_ok(B, Hkv, max_pages, P)) return 0;
    // the lists of moved slots, and their lengths
    return round_up((size_t)B * Hkv * max_pages * P * sizeof(int32_t), 256) +
           round_up((size_t)B * Hkv * sizeof(int32_t), 256) + 256;
}

int kv_evict(const float *weight, const int32_t *position, uint16_t *k_cache, uint16_t *v_cache,
             const int32_t *page_table, const int32_t *kv_len, const int32_t *seen,
             const int32_t *fixed_len, int B, int Hkv, int D, int P, int max_pages, int num_pages,
             int max_kv_len, int budget, int recent, float *weight_out, int32_t *position_out,
             int32_t *kept_len, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!evict_shape_ok(B, Hkv, max_pages, P) || D < 8 || D % 8 != 0 || D > 1024 ||
        num_pages < 1 || max_kv_len < 0 || budget < 0 || recent < 0)
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!weight || !position || !k_cache || !v_cache || !page_table || !kv_len || !seen ||
        !weight_out || !position_out || !kept_len || !workspace)
        return TV_ERR_NULL;
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(workspace)) return TV_ERR_ALIGN;
    if (workspace_bytes < tv_evict_workspace_size(B, Hkv, max_pages, P)) return TV_ERR_WORKSPACE;
    if (!device_ok()) return TV_ERR_DEVICE;
    // one workgroup of a sequence writes its kept length while others read these
    if (overlap(kept_len, kv_len, B) || overlap(kept_len, seen, B) || overlap(kept_len, fixed_len, B))
        return TV_ERR_OVERLAP;
    tv::EvictParams p{};
    p.weight = weight; p.position = position; p.page_table = page_table; p.kv_len = kv_len;
    p.seen = seen; p.fixed_len = fixed_len; p.k_cache = k_cache; p.v_cache = v_cache;
    p.weight_out = weight_out; p.position_out = position_out; p.kept_len = kept_len;
    p.moves = static_cast<int32_t *>(workspace);
    p.count = p.moves + round_up((size_t)B * Hkv * max_pages * P * sizeof(int32_t), 256) / sizeof(int32_t);
    p.B = B; p.Hkv = Hkv; p.D = D; p.p_shift = __builtin_ctz((unsigned)P);
    p.max_pages = max_pages; p.num_pages = num_pages; p.budget = budget; p.recent = recent;
    const long cap = (long)max_pages * P;
    p.max_keys = (int)(max_kv_len < cap ? max_kv_len : cap);
    return tv::launch_evict(p, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

size_t tv_window_attention_workspace_size(int B, int N, int Hq, int Hkv, int D) {
    if (!attn_shape_ok(B, N, Hq, Hkv, D)) return 0;
    return attn_workspace(attn_shape(N, Hq, Hkv), D, cu_count() * kWgPerCu, true).total;
}

int tree_verify_attention_window(const uint16_t *q, const uint16_t *k_tree, const uint16_t *v_tree,
                                 const uint16_t *k_cache, const uint16_t *v_cache, const int32_t *page_table,
                                 const int32_t *kv_len, const int32_t *parent, const int32_t *num_nodes, int B, int N,
                                 int Hq, int Hkv, int D, int P, int max_pages, int num_pages, int max_kv_len,
                                 int window, int sinks, float scale, uint16_t *out, float *lse, void *workspace,
                                 size_t workspace_bytes, hipStream_t stream) {
    if (!window_shape_ok(B, N, Hq, Hkv, D, P, max_pages, num_pages, max_kv_len, window, sinks)) return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!q || !k_tree || !v_tree || !k_cache || !v_cache || !page_table || !kv_len || !parent || !out || !workspace)
        return TV_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(k_cache) || !aligned16(v_cache) ||
        !aligned16(out) || !aligned16(workspace))
        return TV_ERR_ALIGN;
    const AttnShape s = attn_shape(N, Hq, Hkv);
    const int max_wg = cu_count() * kWgPerCu;
    const AttnWorkspace ws = attn_workspace(s, D, max_wg, true);
    if (workspace_bytes < ws.total) return TV_ERR_WORKSPACE;
    const long max_len = (long)max_pages * P;
    if (attn_tiles(s, B, Hkv, max_len) >= kMaxTiles) return TV_ERR_SHAPE;
    if (!device_ok()) return TV_ERR_DEVICE;

    tv::WindowAttnParams p{};
    window_params(p, q, k_tree, v_tree, page_table, kv_len, parent, num_nodes, B, N, Hq, Hkv, D, P, max_pages, num_pages,
                  window, sinks, scale, out, lse, workspace, ws);
    p.k_cache = k_cache; p.v_cache = v_cache;
    // the launch of tree_verify_attention over as many tiles as the window leaves
    const long tiles = window_tiles(max_kv_len < max_len ? max_kv_len : max_len, window, sinks);
    long num_wg = attn_tiles(s, B, Hkv, tiles * tv::kKeyTile) / kMinShareTiles;
    if (num_wg < 1) num_wg = 1;
    if (num_wg > max_wg) num_wg = max_wg;
    const bool small_pages = P < 1024 / (2 * D);
    const bool whole = whole_units(s, B, N, Hkv, D, tiles, small_pages, max_wg);
    if (whole) num_wg = (long)B * Hkv * s.row_blocks;
    p.rows_per_block = s.rows_per_block;
    p.setup_tiles = kSetupTiles;
    p.small_pages = small_pages ? 1 : 0;
    p.narrow = s.rows <= 16 ? 1 : 0;
    p.num_wg = (int)num_wg;
    p.whole_units = whole ? 1 : 0;
    return tv::launch_window_attention(p, D, s.waves, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

size_t tv_kv4_attention_workspace_size(int B, int N, int Hq, int Hkv, int D) {
    if (!attn_shape_ok(B, N, Hq, Hkv, D)) return 0;
    size_t need = 0;                                // of either kernel: lengths and tables choose
    for (bool stream : {false, true}) {
        const Kv4Shape s = kv4_shape(N, Hq, Hkv, stream);
        const size_t n = attn_workspace(s, D, s.max_wg, true).total;
        if (need < n && (!stream || s.rows <= kv4_stream_rows(LONG_MAX))) need = n;
    }
    return need;
}

int tree_verify_attention_kv4(const uint16_t *q, const uint16_t *k_tree, const uint16_t *v_tree, const uint8_t *k4,
                              const uint8_t *v4, const uint8_t *scales, const int32_t *page_table,
                              const int32_t *kv_len, const int32_t *parent, const int32_t *num_nodes, int B, int N,
                              int Hq, int Hkv, int D, int P, int max_pages, int num_pages, int max_kv_len, int window,
                              int sinks, float scale, uint16_t *out, float *lse, void *workspace,
                              size_t workspace_bytes, hipStream_t stream) {
    if (!window_shape_ok(B, N, Hq, Hkv, D, P, max_pages, num_pages, max_kv_len, window, sinks)) return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!q || !k_tree || !v_tree || !k4 || !v4 || !scales || !page_table || !kv_len || !parent || !out || !workspace)
        return TV_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_tree) || !aligned16(v_tree) || !aligned16(k4) || !aligned16(v4) ||
        !aligned16(scales) || !aligned16(out) || !aligned16(workspace))
        return TV_ERR_ALIGN;
    if (workspace_bytes < tv_kv4_attention_workspace_size(B, N, Hq, Hkv, D)) return TV_ERR_WORKSPACE;
    const long max_len = (long)max_pages * P;
    const long tiles = window_tiles(max_kv_len < max_len ? max_kv_len : max_len, window, sinks);
    // what the window call accepts; where the lengths that the table has room for are too many
    // tiles in blocks of few rows, larger blocks are taken
    const AttnShape plain = attn_shape(N, Hq, Hkv);
    if (attn_tiles(plain, B, Hkv, max_len) >= kMaxTiles) return TV_ERR_SHAPE;
    Kv4Shape s = kv4_shape(N, Hq, Hkv, plain.rows <= kv4_stream_rows(tiles * tv::kKeyTile));
    if (s.stream && kv4_tiles(s, B, Hkv, (max_len + tv::kKeyTile - 1) / tv::kKeyTile) >= kMaxTiles)
        s = kv4_shape(N, Hq, Hkv, false);
    const AttnWorkspace ws = attn_workspace(s, D, s.max_wg, true);
    if (!device_ok()) return TV_ERR_DEVICE;

    tv::Kv4AttnParams p{};
    window_params(p, q, k_tree, v_tree, page_table, kv_len, parent, num_nodes, B, N, Hq, Hkv, D, P, max_pages, num_pages,
                  window, sinks, scale, out, lse, workspace, ws);
    p.k4 = k4; p.v4 = v4; p.scales = scales;
    p.g_inv = s.G == 1 ? 0u : (unsigned)((1ull << 32) / (unsigned)s.G + 1);
    long num_wg = kv4_tiles(s, B, Hkv, tiles) / (s.stream ? kKv4StreamMinShareTiles : kMinShareTiles);
    if (num_wg < 1) num_wg = 1;
    if (num_wg > s.max_wg) num_wg = s.max_wg;
    p.rows_per_block = s.rows_per_block;
    p.setup_tiles = s.setup;
    p.num_wg = (int)num_wg;
    return tv::launch_kv4_attention(p, D, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

int kv4_write(const uint16_t *k, const uint16_t *v, uint8_t *k4, uint8_t *v4, uint8_t *scales,
              const int32_t *page_table, const int32_t *start, const int32_t *idx, const int32_t *count, int B, int T,
              int Hkv, int D, int P, int max_pages, int num_pages, uint16_t *k_held, uint16_t *v_held,
              hipStream_t stream) {
    if (B < 0 || B > 65535 || T < 0 || Hkv < 1 || (D != 64 && D != 128) || !pow2(P) || P > 256 || max_pages < 1 ||
        num_pages < 1 || (long)max_pages * P >= (1l << 31))
        return TV_ERR_SHAPE;
    // workgroups of 256 threads per sequence: fewer than 2^32 threads
    if (((long)T + 15) / 16 * Hkv >= (1l << 24)) return TV_ERR_SHAPE;
    if (B == 0 || T == 0) return TV_OK;
    if (!k || !v || !k4 || !v4 || !scales || !page_table || !start) return TV_ERR_NULL;
    if (!aligned16(k) || !aligned16(v) || !aligned16(k4) || !aligned16(v4) || !aligned16(scales) ||
        !aligned16(k_held) || !aligned16(v_held))
        return TV_ERR_ALIGN;
    // held rows may take their own rows' place, which the thread that writes has read; no others'
    const size_t bytes = (size_t)B * T * Hkv * D * sizeof(uint16_t);
    auto meet = [&](const uint16_t *x, const uint16_t *y) {
        const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
        return x && y && (a < b ? b - a : a - b) < bytes;
    };
    if (meet(k_held, v) || meet(v_held, k) || meet(k_held, v_held) || (meet(k_held, k) && (idx || k_held != k)) ||
        (meet(v_held, v) && (idx || v_held != v)))
        return TV_ERR_OVERLAP;
    if (!device_ok()) return TV_ERR_DEVICE;
    tv::Kv4WriteParams p;
    p.k = k; p.v = v; p.k4 = k4; p.v4 = v4; p.scales = scales; p.page_table = page_table; p.start = start;
    p.idx = idx; p.count = count; p.k_held = k_held; p.v_held = v_held;
    p.T = T; p.Hkv = Hkv; p.p_shift = __builtin_ctz((unsigned)P); p.max_pages = max_pages; p.num_pages = num_pages;
    return tv::launch_kv4_write(p, B, D, stream) == hipSuccess ? TV_OK : TV_ERR_HIP;
}

int tv_validate_inputs(const int32_t *page_table, const int32_t *kv_len, const int32_t *parent,
                       const int32_t *num_nodes, int B, int N, int P, int max_pages,
                       int num_pages, int32_t *status_word, hipStream_t stream) {
    if (B < 0 || N < 1 || N > tv::kMaxNodes || !pow2(P) || max_pages < 1 || num_pages < 1)
        return TV_ERR_SHAPE;
    if (!status_word || (B > 0 && (!page_table || !kv_len || !parent))) return TV_ERR_NULL;
    if (!device_ok()) return TV_ERR_DEVICE;
    const hipError_t e = tv::launch_validate(page_table, kv_len, parent, num_nodes, B, N, P,
                                             max_pages, num_pages, status_word, stream);
    return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

static bool tree_build_shape_ok(int B, int S, int V, int H, int k) {
    return B >= 0 && B <= 65535 && S >= 1 && S <= tv::kTbMaxSteps && V >= 1 && H >= 0 &&
           H <= V && k >= 1 && k <= tv::kTbMaxK && k <= V;
}

size_t tv_tree_build_workspace_size(int B, int S, int V, int H, int k) {
    if (!tree_build_shape_ok(B, S, V, H, k)) return 0;
    return tv::tree_build_plan(B, S, V, H, k).bytes;
}

int tree_build(const float *logits, const int32_t *root_token, const uint16_t *token_info,
               const int32_t *hot_vocab, const int32_t *hot_index, int B, int S, int V, int H,
               int k, int budget, int32_t *parent, int32_t *token, float *joint,
               int32_t *num_nodes, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!tree_build_shape_ok(B, S, V, H, k) || budget < 1 || budget > tv::kMaxNodes)
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!logits || !root_token || !parent || !token || !joint || !num_nodes || !workspace ||
        (H > 0 && (!token_info || !hot_vocab || !hot_index)))
        return TV_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(logits) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 7u))
        return TV_ERR_ALIGN;
    if (workspace_bytes < tv_tree_build_workspace_size(B, S, V, H, k)) return TV_ERR_WORKSPACE;
    if (!device_ok()) return TV_ERR_DEVICE;
    const hipError_t e = tv::launch_tree_build(logits, root_token, token_info, hot_vocab,
                                               hot_index, nullptr, 0, B, S, V, H, k, budget,
                                               parent, token, joint, num_nodes, workspace,
                                               stream);
    return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

int tree_resample(const float *logits, const int32_t *bonus_token, const int32_t *accept_len,
                  const uint16_t *token_info, const int32_t *hot_vocab, const int32_t *hot_index,
                  int B, int S, int V, int H, int k, int r, int budget, int32_t *parent,
                  int32_t *token, float *joint, int32_t *num_nodes, void *workspace,
                  size_t workspace_bytes, hipStream_t stream) {
    if (!tree_build_shape_ok(B, S, V, H, k) || budget < 1 || budget > tv::kMaxNodes || r < 0)
        return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!logits || !bonus_token || !accept_len || !parent || !token || !joint || !num_nodes ||
        !workspace || (H > 0 && (!token_info || !hot_vocab || !hot_index)))
        return TV_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(logits) & 3u) || (reinterpret_cast<uintptr_t>(workspace) & 7u))
        return TV_ERR_ALIGN;
    if (workspace_bytes < tv_tree_build_workspace_size(B, S, V, H, k)) return TV_ERR_WORKSPACE;
    if (!device_ok()) return TV_ERR_DEVICE;
    const hipError_t e = tv::launch_tree_build(logits, bonus_token, token_info, hot_vocab,
                                               hot_index, accept_len, r, B, S, V, H, k, budget,
                                               parent, token, joint, num_nodes, workspace,
                                               stream);
    return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

static bool lm_head_shape_ok(int B, int N, int V, int d) {
    // V: vocabulary ids of a tile's rows (v0 + 0..255) must fit an int
    if (B < 0 || B > 65535 || N < 1 || N > tv::kMaxNodes || V < 1 || V > 0x7FFFFFFF - 256 ||
        d < 64 || d % 64 != 0)
        return false;
    const long long rblocks = ((long long)B * N + 255) / 256;
    const long long groups = ((long long)tv::lm_head_vocab_tiles(V) + 7) / 8 * 8 * rblocks;
    return groups <= 0x7FFFFFFFll - 256;         // a workgroup's next tile (256 further on) fits an int
}

size_t tv_lm_head_workspace_size(int B, int N, int V, int d) {
    if (!lm_head_shape_ok(B, N, V, d)) return 0;
    return round_up((size_t)B * N * sizeof(unsigned long long), 256) + 256;
}

int tree_lm_head_argmax_accept(const uint16_t *hidden, const uint16_t *w_head,
                               const int32_t *draft_tokens, const int32_t *parent,
                               const int32_t *num_nodes, int B, int N, int V, int d,
                               int32_t *argmax_out, int32_t *accept_len, int32_t *accept_idx,
                               int32_t *bonus_token, void *workspace, size_t workspace_bytes,
                               hipStream_t stream) {
    if (!lm_head_shape_ok(B, N, V, d)) return TV_ERR_SHAPE;
    if (B == 0) return TV_OK;
    if (!hidden || !w_head || !draft_tokens || !parent || !argmax_out || !accept_len ||
        !accept_idx || !bonus_token || !workspace)
        return TV_ERR_NULL;
    if (!aligned16(hidden) || !aligned16(w_head) || (reinterpret_cast<uintptr_t>(workspace) & 7u))
        return TV_ERR_ALIGN;
    if (workspace_bytes < tv_lm_head_workspace_size(B, N, V, d)) return TV_ERR_WORKSPACE;
    if (!device_ok()) return TV_ERR_DEVICE;
    const hipError_t e = tv::launch_lm_head_argmax_accept(
        hidden, w_head, draft_tokens, parent, num_nodes, B, N, V, d, argmax_out, accept_len,
        accept_idx, bonus_token, static_cast<unsigned long long *>(workspace), stream);
    return e == hipSuccess ? TV_OK : TV_ERR_HIP;
}

}  // extern "C"
