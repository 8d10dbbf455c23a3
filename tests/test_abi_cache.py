"""Host-side argument checks of the cache operators (CPU only; no kernel is
ever launched, no pointer is dereferenced), and of their Python wrappers."""
import ctypes
import os

import pytest
import torch

FAKE = ctypes.c_void_p(0x10000)
NULL = ctypes.c_void_p(0)
STREAM = ctypes.c_void_p(0)
ODD = ctypes.c_void_p(0x10008)


@pytest.fixture(scope="module")
def lib():
    from paper_2602_21224_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2602_21224_amd import build
        build.build()
    return _lib.load()


def shared(lib, **kw):
    a = dict(q=FAKE, k_tree=FAKE, v_tree=FAKE, k_cache=FAKE, v_cache=FAKE, page_table=FAKE,
             kv_len=FAKE, parent=FAKE, num_nodes=NULL, group_start=FAKE, shared_len=FAKE, groups=1, B=2,
             N=8, Hq=8, Hkv=2, D=128, P=16, max_pages=4, num_pages=8, max_kv_len=32, scale=0.0, out=FAKE,
             lse=NULL, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return lib.tree_verify_attention_shared(*a.values(), STREAM)


def test_shared_attention_argument_checks(lib):
    assert shared(lib, B=0) == 0
    assert shared(lib, q=NULL) == -1 and shared(lib, ws=NULL) == -1
    assert shared(lib, group_start=NULL) == -1 and shared(lib, shared_len=NULL) == -1
    assert shared(lib, groups=-1) == -2 and shared(lib, groups=257) == -2
    assert shared(lib, B=513) == -2 and shared(lib, B=-1) == -2
    assert shared(lib, D=96) == -2 and shared(lib, N=257) == -2 and shared(lib, Hq=6, Hkv=4) == -2
    assert shared(lib, P=12) == -2 and shared(lib, max_pages=0) == -2 and shared(lib, max_kv_len=-1) == -2
    assert shared(lib, max_pages=1 << 30) == -2
    assert shared(lib, v_cache=ODD) == -3 and shared(lib, out=ODD) == -3
    need = lib.tv_shared_attention_workspace_size(2, 8, 8, 2, 128, 1)
    assert need > 0 and shared(lib, ws_bytes=need - 1) == -4
    many = dict(B=512, N=256, Hq=1025, Hkv=1025, ws_bytes=1 << 62)        # more than 2^34 output values
    assert shared(lib, **many) == -2 and shared(lib, **{**many, "Hq": 1024, "Hkv": 1024, "q": NULL}) == -1
    assert lib.tv_shared_attention_workspace_size(512, 256, 1025, 1025, 128, 1) == 0
    # well-formed on a machine without a GPU: stops at the device check, launches nothing
    assert shared(lib) in (-4, -6)
    assert shared(lib, groups=0, group_start=NULL, shared_len=NULL) in (-4, -6)
    for bad in ((513, 8, 8, 2, 128, 1), (2, 8, 8, 2, 96, 1), (2, 8, 8, 2, 128, 257), (2, 8, 8, 2, 128, -1)):
        assert lib.tv_shared_attention_workspace_size(*bad) == 0


def weights(lib, **kw):
    a = dict(q=FAKE, lse=FAKE, k_cache=FAKE, page_table=FAKE, kv_len=FAKE, idx=FAKE, alen=FAKE, seen=FAKE,
             fixed=NULL, weight=FAKE, B=2, N=8, Hq=8, Hkv=2, D=128, P=16, max_pages=4, num_pages=8,
             max_kv_len=32, scale=0.0, weight_out=FAKE, position=FAKE)
    a.update(kw)
    return lib.kv_accumulate_weights(*a.values(), STREAM)


def test_weight_argument_checks(lib):
    assert weights(lib, B=0) == 0
    for name in ("q", "lse", "k_cache", "page_table", "kv_len", "idx", "alen", "seen", "weight", "weight_out",
                 "position"):
        assert weights(lib, **{name: NULL}) == -1, name
    assert weights(lib, D=80) == -2 and weights(lib, N=0) == -2 and weights(lib, Hq=7, Hkv=2) == -2
    assert weights(lib, Hq=64, Hkv=2, N=128) == -2                # more than 2048 rows per KV head
    assert weights(lib, B=65536) == -2 and weights(lib, P=0) == -2 and weights(lib, num_pages=0) == -2
    assert weights(lib, max_pages=(1 << 20) + 1) == -2             # more than 2^24 slots
    assert weights(lib, q=ODD) == -3 and weights(lib, k_cache=ODD) == -3
    assert weights(lib) == -6 and weights(lib, fixed=FAKE) == -6


def evict(lib, **kw):
    a = dict(weight=FAKE, position=FAKE, k_cache=FAKE, v_cache=FAKE, page_table=FAKE, kv_len=FAKE, seen=FAKE,
             fixed=NULL, B=2, Hkv=2, D=128, P=16, max_pages=4, num_pages=8, max_kv_len=32, budget=20,
             recent=4, weight_out=FAKE, position_out=FAKE, kept=FAKE, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return lib.kv_evict(*a.values(), STREAM)


def test_evict_argument_checks(lib):
    assert evict(lib, B=0) == 0
    for name in ("weight", "position", "k_cache", "v_cache", "page_table", "kv_len", "seen", "weight_out",
                 "position_out", "kept", "ws"):
        assert evict(lib, **{name: NULL}) == -1, name
    assert evict(lib, budget=-1) == -2 and evict(lib, recent=-1) == -2
    assert evict(lib, D=4) == -2 and evict(lib, D=100) == -2 and evict(lib, D=1032) == -2
    assert evict(lib, P=24) == -2 and evict(lib, Hkv=0) == -2 and evict(lib, max_pages=(1 << 20) + 1) == -2
    assert evict(lib, v_cache=ODD) == -3 and evict(lib, ws=ODD) == -3
    need = lib.tv_evict_workspace_size(2, 2, 4, 16)
    assert need > 0 and evict(lib, ws_bytes=need - 1) == -4
    assert evict(lib) == -6 and evict(lib, fixed=FAKE) == -6
    assert lib.tv_evict_workspace_size(2, 2, 4, 3) == 0 and lib.tv_evict_workspace_size(-1, 2, 4, 16) == 0


def test_wrappers_refuse_tensors_that_are_not_on_the_gpu(lib):
    import paper_2602_21224_amd as T
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(ValueError, match="on the GPU"):
        T.tree_verify_attention_shared(bf(1, 1, 2, 64), bf(1, 1, 2, 64), bf(1, 1, 2, 64), bf(1, 1, 2, 64),
                                       bf(1, 1, 2, 64), i32(1, 1), i32(1), i32(1, 1), i32(2), i32(1),
                                       max_kv_len=1)
    with pytest.raises(ValueError, match="on the GPU"):
        T.kv_accumulate_weights(bf(1, 1, 2, 64), torch.zeros(1, 1, 2), bf(1, 1, 2, 64), i32(1, 1), i32(1),
                                i32(1, 1), i32(1), torch.zeros(1, 2, 1), i32(1, 2, 1), i32(1), max_kv_len=1)
    with pytest.raises(ValueError, match="on the GPU"):
        T.kv_evict(torch.zeros(1, 2, 1), i32(1, 2, 1), bf(1, 1, 2, 64), bf(1, 1, 2, 64), i32(1, 1), i32(1),
                   i32(1), max_kv_len=1, budget=1)
