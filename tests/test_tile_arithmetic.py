"""The attention kernels' arithmetic on tiles and positions, compiled for the host from
their own headers (CPU only)."""
import ctypes
import os
import random
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_21224_amd", "csrc")
KEYS, CACHED = 64, 512                 # keys per tile, page ids per window
LONGEST = 0x7FFFFFFF - 1024            # tokens of the longest prefix

SOURCE = """
#include "tree_attention_common.h"
#define API extern "C" __attribute__((visibility("default")))
API int page_window_end(int first, int p_shift) { return tv::page_window_end(first, p_shift); }
API int clamp_len(int L, int max_pages, int p_shift) {
    tv::AttnParams p{};
    p.max_pages = max_pages;
    p.p_shift = p_shift;
    return tv::clamp_len(L, p);
}
typedef unsigned long long Set[4];
API void span(int L, int window, int sinks, int *lo_ns_gap) {
    tv::WindowAttnParams p{};
    p.window = window;
    p.sinks = sinks;
    const tv::Span s = tv::span_of(L, p);
    lo_ns_gap[0] = s.lo;
    lo_ns_gap[1] = s.ns;
    lo_ns_gap[2] = s.gap;
}
API int window_clear(int L, int window, int sinks, int base, int N) {
    tv::WindowAttnParams p{};
    p.window = window;
    p.sinks = sinks;
    return tv::window_clear(tv::span_of(L, p), base, N);
}
API unsigned long long window_bits(int L, int window, int sinks, int base, const Set &anc) {
    tv::WindowAttnParams p{};
    p.window = window;
    p.sinks = sinks;
    return tv::window_bits(tv::span_of(L, p), base, anc);
}
API unsigned long long window_path(int L, int window, int sinks, const Set &anc, int word) {
    tv::WindowAttnParams p{};
    p.window = window;
    p.sinks = sinks;
    return tv::window_path(anc, word, L, p);
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    from paper_2602_21224_amd import build
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("tiles")
    src, out = d / "tiles.hip", d / "libtiles.so"
    src.write_text(SOURCE)
    flags = [f for f in build.FLAGS if f != "-O3"]
    subprocess.run([build.HIPCC, *flags, "-O1", "--offload-host-only", "-I", CSRC, "-shared", str(src), "-o",
                    str(out)], check=True, capture_output=True)
    h = ctypes.CDLL(str(out))
    h.window_bits.restype = h.window_path.restype = ctypes.c_uint64
    return h


def node_set(nodes):
    """A node's ancestor set, itself included, as four words."""
    bits = sum(1 << i for i in nodes)
    return (ctypes.c_uint64 * 4)(*[(bits >> 64 * w) & (1 << 64) - 1 for w in range(4)])


@pytest.mark.parametrize("shift", range(9))
@pytest.mark.parametrize("back", [1, 64, 100000, 131072, 200000])
def test_sub_ranges_of_a_piece_reach_its_end(host, shift, back):
    """A piece's tiles are taken in sub-ranges whose pages fit the table of page ids: each
    begins where the last one ended and takes whole tiles, up to the longest prefix."""
    P = 1 << shift
    L = LONGEST // P * P
    tiles = -(-L // KEYS)
    for t0 in (max(tiles - 1 - back // KEYS, 0), tiles - 1):
        t = t0
        while t < tiles:
            first = t * KEYS >> shift
            end = host.page_window_end(first, shift)
            assert end == (first + CACHED) * P // KEYS and end > t
            t = min(end, tiles)


@pytest.mark.parametrize("shift", range(9))
def test_lengths_are_those_of_the_table_whatever_its_size(host, shift):
    """A table may have room for more tokens than a prefix can have."""
    for columns in (1, 3, (LONGEST >> shift) + 1, (1 << 31 - shift) - 1, 1 << 31 - shift, (1 << 32 - shift) + 5,
                    (1 << 31) - 1):
        if columns >= 1 << 31:
            continue
        room = min(columns << shift, LONGEST)
        for L in (-5, 0, 1, 7, 300, 0x7FFFFFC0, 0x7FFFFFFF, LONGEST, LONGEST + 1):
            assert host.clamp_len(L, columns, shift) == min(max(L, 0), room), (columns, L)


WINDOWS = [(1, 0), (1, 3), (5, 64), (63, 1), (64, 0), (64, 65), (65, 130), (100, 63), (129, 4), (200, 300), (0x7FFFFFFF, 9)]
LENGTHS = list(range(0, 70)) + [127, 128, 129, 191, 192, 193, 200, 255, 256, 257, 300, 319, 320, 321, 384, 447, 448, 500]


@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_tiles_and_masks_of_a_window_are_its_definition(host, window, sinks):
    """Position t of the prefix is seen from depth d iff t < sinks or t > L + d - window."""
    N = 40
    chains = {d: node_set(range(d + 1)) for d in (0, 1, 2, 7, 39)}
    out = (ctypes.c_int * 3)()
    for L in LENGTHS:
        host.span(L, window, sinks, out)
        lo, ns, gap = out
        assert lo == max(L - window + 1, 0)
        for t in range(-(-L // KEYS)):
            base = t * KEYS
            for d, anc in chains.items():
                want = sum(1 << i for i in range(KEYS) if base + i < sinks or base + i > L + d - window)
                inside = (1 << min(L - base, KEYS)) - 1
                if ns <= t < ns + gap:
                    assert want & inside == 0, (L, t, d)
                elif host.window_clear(L, window, sinks, base, N):
                    assert want & inside == inside, (L, t, d)
                else:
                    assert host.window_bits(L, window, sinks, base, anc) & inside == want & inside, (L, t, d)


@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_tiles_before_the_window_need_no_root_paths(host, window, sinks):
    """A piece of work without them has whatever was there before in their place."""
    for L in LENGTHS:
        for base in range(0, L, KEYS):
            if base + KEYS <= L - window + 1:
                want = sum(1 << i for i in range(KEYS) if base + i < sinks)
                for stale in (node_set([]), node_set([0]), node_set(range(256))):
                    assert host.window_bits(L, window, sinks, base, stale) == want, (L, base)


@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_root_paths_inside_a_window(host, window, sinks):
    rng = random.Random(window + sinks)
    for L in (0, 1, 3, 60, 64, 298, 299, 500):
        nodes = sorted(rng.sample(range(256), rng.choice([1, 2, 30, 200, 255])))
        anc = node_set(nodes)
        at = L + len(nodes) - 1
        want = sum(1 << i for d, i in enumerate(nodes) if L + d < sinks or L + d > at - window)
        for word in range(4):
            assert host.window_path(L, window, sinks, anc, word) == (want >> 64 * word) & (1 << 64) - 1


@pytest.mark.parametrize("source", ["tree_attention_kv4.hip", "tree_attention_kv4_wide.hip"])
def test_the_scan_of_lengths_counts_the_units_that_the_search_walks(source, tmp_path):
    """Over 4 bits the cumulative tiles of a batch come from the function whose terms the
    search for a piece adds up: without it the kernels do not compile."""
    from paper_2602_21224_amd import build
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    shutil.copytree(CSRC, tmp_path / "csrc", ignore=shutil.ignore_patterns("*.so", "*.o"))
    header = tmp_path / "csrc" / "tree_attention_kv4.h"
    text, found = re.subn(r"\{\s*return p\.Hkv \* head_tiles\([^;]*;\s*\}", "= delete;", header.read_text())
    assert found == 1
    cmd = [build.HIPCC, *[f for f in build.FLAGS if f != "-O3"], "-fsyntax-only", "--offload-host-only",
           str(tmp_path / "csrc" / source)]
    with_it = subprocess.run(cmd, capture_output=True, text=True)
    assert with_it.returncode == 0, with_it.stderr[-2000:]
    header.write_text(text)
    without = subprocess.run(cmd, capture_output=True, text=True)
    assert without.returncode != 0 and "deleted function" in without.stderr
