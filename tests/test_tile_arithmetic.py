"""The attention kernels' arithmetic on tiles and positions, compiled for the host from
their own headers (CPU only)."""
import ctypes
import os
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
    return ctypes.CDLL(str(out))


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
