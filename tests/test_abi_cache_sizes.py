"""Sizes of the shared-prefix attention: what tree_verify_attention accepts is accepted
(CPU only; the calls stop at the device check)."""
import pytest

from tests.test_abi_cache import lib, shared  # noqa: F401  (lib is a fixture)


def plain_tiles(B, N, Hq, Hkv, tokens):
    """Tiles of tree_verify_attention's launch, of which it takes fewer than 2^30: per row
    block of 128 or 256 rows three, the prefix's, and those of the tree up to its last row."""
    G = Hq // Hkv
    rows, block = N * G, 256 if N * G > 128 else 128
    ends = [min(r + block, rows) for r in range(0, rows, block)]
    return B * Hkv * sum(3 + -(-tokens // 64) + -(-((end - 1) // G + 1) // 64) for end in ends)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("groups", [0, 1, 7])
@pytest.mark.parametrize("B,N,Hq,Hkv", [(512, 1, 32, 32), (512, 1, 256, 32), (512, 12, 32, 32), (512, 24, 32, 8),
                                        (512, 64, 32, 8), (64, 48, 8, 8), (16, 256, 64, 8), (1, 1, 1, 1)])
def test_what_the_plain_call_accepts_is_accepted(lib, B, N, Hq, Hkv, D, groups):  # noqa: F811
    for shift in range(4, 26):           # tables of 2^8 to 2^29 tokens a sequence
        if plain_tiles(B, N, Hq, Hkv, 16 << shift) < 1 << 30:
            assert shared(lib, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, groups=groups, max_pages=1 << shift,
                          max_kv_len=1 << 26, ws_bytes=1 << 62) == -6, shift


@pytest.mark.parametrize("groups", [0, 1])
def test_more_tiles_than_can_be_counted_are_refused(lib, groups):  # noqa: F811
    big = dict(B=512, N=64, Hq=32, Hkv=8, groups=groups, max_kv_len=1 << 26, ws_bytes=1 << 62)
    assert shared(lib, max_pages=1 << 20, **big) == -2


def test_tables_of_two_to_the_31_tokens_are_refused(lib):  # noqa: F811
    one = dict(B=1, N=1, Hq=1, Hkv=1, D=64, P=256, ws_bytes=1 << 62)
    assert shared(lib, max_pages=(1 << 23) - 1, **one) == -6
    assert shared(lib, max_pages=1 << 23, **one) == -2
