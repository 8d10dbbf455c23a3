"""Host-side argument checks of the long-context operators (CPU only; no kernel is ever
launched, no pointer is dereferenced), and of their Python wrappers."""
import ctypes

import pytest
import torch

from tests.test_abi_cache import FAKE, NULL, ODD, STREAM, lib  # noqa: F401  (lib is a fixture)

BIG = 1 << 62


def window(lib, **kw):  # noqa: F811
    a = dict(q=FAKE, k_tree=FAKE, v_tree=FAKE, k_cache=FAKE, v_cache=FAKE, page_table=FAKE, kv_len=FAKE, parent=FAKE,
             num_nodes=NULL, B=2, N=8, Hq=8, Hkv=2, D=128, P=16, max_pages=4, num_pages=8, max_kv_len=32, window=20,
             sinks=4, scale=0.0, out=FAKE, lse=NULL, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    return lib.tree_verify_attention_window(*a.values(), STREAM)


def kv4(lib, **kw):  # noqa: F811
    a = dict(q=FAKE, k_tree=FAKE, v_tree=FAKE, k4=FAKE, v4=FAKE, scales=FAKE, page_table=FAKE, kv_len=FAKE, parent=FAKE,
             num_nodes=NULL, B=2, N=8, Hq=8, Hkv=2, D=128, P=16, max_pages=4, num_pages=8, max_kv_len=32, window=20,
             sinks=4, scale=0.0, out=FAKE, lse=NULL, ws=FAKE, ws_bytes=BIG)
    a.update(kw)
    return lib.tree_verify_attention_kv4(*a.values(), STREAM)


@pytest.mark.parametrize("call,cache,size", [(window, ("k_cache", "v_cache"), "tv_window_attention_workspace_size"),
                                             (kv4, ("k4", "v4", "scales"), "tv_kv4_attention_workspace_size")])
def test_attention_argument_checks(lib, call, cache, size):  # noqa: F811
    assert call(lib, B=0) == 0 and call(lib, B=0, q=NULL) == 0
    for name in ("q", "k_tree", "v_tree", "page_table", "kv_len", "parent", "out", "ws") + cache:
        assert call(lib, **{name: NULL}) == -1, name
    assert call(lib, B=-1) == -2 and call(lib, B=1025) == -2
    assert call(lib, D=96) == -2 and call(lib, N=0) == -2 and call(lib, N=257) == -2
    assert call(lib, Hq=6, Hkv=4) == -2 and call(lib, Hq=0) == -2 and call(lib, Hkv=0) == -2
    assert call(lib, Hq=64, Hkv=2, N=128) == -2                    # more than 2048 rows per KV head
    for P in (0, 12, 512, -16):
        assert call(lib, P=P) == -2, P
    assert call(lib, max_pages=0) == -2 and call(lib, num_pages=0) == -2 and call(lib, max_kv_len=-1) == -2
    assert call(lib, window=-1) == -2 and call(lib, sinks=-1) == -2
    one = dict(B=1, N=1, Hq=1, Hkv=1, D=64, P=1)
    assert call(lib, **one, max_pages=0x7FFFFFFF - 1024) in (-6, 0)         # the longest table
    assert call(lib, **one, max_pages=0x7FFFFFFF - 1023) == -2
    assert call(lib, B=1024, Hkv=64, Hq=64, P=256, max_pages=1 << 20) == -2  # more tiles than are counted
    for name in ("q", "k_tree", "v_tree", "out", "ws") + cache:
        assert call(lib, **{name: ODD}) == -3, name
    need = getattr(lib, size)(2, 8, 8, 2, 128)
    assert need > 0 and call(lib, ws_bytes=need - 1) == -4 and call(lib, ws_bytes=need) == -6
    # well-formed on a machine without a GPU: stops at the device check, launches nothing
    assert call(lib) == -6 and call(lib, num_nodes=FAKE, lse=FAKE, window=0, sinks=0) == -6
    assert call(lib, window=0x7FFFFFFF, sinks=0x7FFFFFFF, max_kv_len=0x7FFFFFFF) == -6
    for bad in ((1025, 8, 8, 2, 128), (2, 8, 8, 2, 96), (2, 0, 8, 2, 128), (2, 8, 8, 3, 128)):
        assert getattr(lib, size)(*bad) == 0


def write(lib, **kw):  # noqa: F811
    a = dict(k=FAKE, v=ctypes.c_void_p(0x20000), k4=FAKE, v4=FAKE, scales=FAKE, page_table=FAKE, start=FAKE, idx=NULL,
             count=NULL, B=2, T=5, Hkv=2, D=128, P=16, max_pages=4, num_pages=8, k_held=NULL, v_held=NULL)
    a.update(kw)
    return lib.kv4_write(*a.values(), STREAM)


def test_write_argument_checks(lib):  # noqa: F811
    at = ctypes.c_void_p
    assert write(lib, B=0) == 0 and write(lib, T=0, k=NULL) == 0
    for name in ("k", "v", "k4", "v4", "scales", "page_table", "start"):
        assert write(lib, **{name: NULL}) == -1, name
    assert write(lib, B=-1) == -2 and write(lib, B=65536) == -2 and write(lib, T=-1) == -2 and write(lib, Hkv=0) == -2
    assert write(lib, D=96) == -2 and write(lib, D=32) == -2 and write(lib, P=3) == -2 and write(lib, P=512) == -2
    assert write(lib, max_pages=0) == -2 and write(lib, num_pages=0) == -2 and write(lib, max_pages=1 << 27) == -2
    assert write(lib, T=1 << 28, Hkv=1) == -2 and write(lib, T=(1 << 28) - 16, Hkv=1) == -6
    assert write(lib, T=1, Hkv=1 << 24) == -2
    for name in ("k", "v", "k4", "v4", "scales", "k_held", "v_held"):
        assert write(lib, **{name: ODD}) == -3, name
    # held rows over their own rows, unless an index moves them; nowhere else over inputs or each other
    far = dict(k_held=at(0x30000), v_held=at(0x40000))
    assert write(lib, **far) == -6 and write(lib, idx=FAKE, count=FAKE, **far) == -6
    assert write(lib, k_held=FAKE, v_held=at(0x20000)) == -6
    assert write(lib, k_held=FAKE, idx=FAKE) == -8 and write(lib, v_held=at(0x20000), idx=FAKE) == -8
    assert write(lib, k_held=at(0x10010)) == -8 and write(lib, k_held=at(0x20000)) == -8 and write(lib, v_held=FAKE) == -8
    assert write(lib, k_held=at(0x30000), v_held=at(0x30100)) == -8
    assert write(lib) == -6


def test_wrappers_refuse_what_does_not_fit(lib):  # noqa: F811
    import paper_2602_21224_amd as T
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError, match="on the GPU"):
        T.tree_verify_attention_window(bf(1, 1, 2, 64), bf(1, 1, 2, 64), bf(1, 1, 2, 64), bf(1, 1, 2, 64),
                                       bf(1, 1, 2, 64), i32(1, 1), i32(1), i32(1, 1), max_kv_len=1, window=4)
    with pytest.raises(ValueError, match="on the GPU"):
        T.tree_verify_attention_kv4(bf(1, 1, 2, 64), bf(1, 1, 2, 64), bf(1, 1, 2, 64), u8(1, 2, 1, 32), u8(1, 2, 1, 32),
                                    u8(1, 2, 1, 2, 2), i32(1, 1), i32(1), i32(1, 1), max_kv_len=1)
    with pytest.raises(ValueError, match="on the GPU"):
        T.kv4_write(bf(1, 1, 2, 64), bf(1, 1, 2, 64), u8(1, 2, 1, 32), u8(1, 2, 1, 32), u8(1, 2, 1, 2, 2), i32(1, 1),
                    i32(1))
