"""Results and workspaces that the cache operators' wrappers allocate for a call on another
stream: their memory is not in use by work that is still to come on the current one."""
import numpy as np
import pytest
import torch

from tests import cache_util as C
from tests import gpu_util as U
from tests.test_gpu_cache import evict, far_table, upload_state

pytestmark = pytest.mark.gpu

LONG = 20_000_000                        # clocks that the current stream is busy: 8 ms and more


def pending(*sizes):
    """Freed blocks of the current stream that it will still write to."""
    torch.cuda.empty_cache()
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda._sleep(LONG)
    for x in blocks:
        x.fill_(0xFF)


def inputs(seed, far):
    """Arguments of the call, in memory before anything is pending."""
    w = C.shared_workload(seed, B=4, N=16, Hq=16, Hkv=4, D=128, P=16, start=[0, 4], shared=[512], own=(0, 300))
    d = U.upload(w)
    table = far_table(w, d["page_table"]) if far else d["page_table"]
    args = [d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"], table, d["kv_len"], d["parent"],
            U.dev(np.array([0, 4], np.int32)), U.dev(np.array([512], np.int32))]
    return args, dict(max_kv_len=1 << 24 if far else w.max_kv_len)


def same(a, b):
    return all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(a, b))


@pytest.mark.parametrize("far", [False, True])
def test_own_tensors_are_not_the_current_streams(far):
    T = U.require_gpu()
    args, hint = inputs(980, far)
    s = C.cache_state(981, B=3, Hkv=4, D=64, P=16, lens=[900, 700, 40])
    e = upload_state(s)
    copy = lambda: {**e, **{k: e[k].clone() for k in ("k_cache", "v_cache", "weight", "position")}}  # noqa: E731
    want = [t.clone() for t in T.tree_verify_attention_shared(*args, **hint)]
    one = copy()
    want_e = [t.clone() for t in evict(T, s, one, 256, 30)]
    side, two = torch.cuda.Stream(), copy()
    size = T.shared_attention_workspace_size(4, 16, 16, 4, 128, 1)
    torch.cuda.synchronize()
    pending(want[0].nbytes, want[1].nbytes, size)
    got = T.tree_verify_attention_shared(*args, **hint, stream=side)
    torch.cuda.synchronize()
    assert same(got, want)
    pending(want_e[2].nbytes, T.evict_workspace_size(3, 4, s["page_table"].shape[1], 16))
    got_e = evict(T, s, two, 256, 30, stream=side)
    torch.cuda.synchronize()
    assert same(got_e, want_e) and same([two["k_cache"], two["v_cache"]], [one["k_cache"], one["v_cache"]])


def test_results_last_until_the_current_stream_is_done_with_them():
    T = U.require_gpu()
    args, hint = inputs(982, False)
    other = [args[0] * 2, *args[1:]]
    want = T.tree_verify_attention_shared(*args, **hint)[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, lse = T.tree_verify_attention_shared(*args, **hint, stream=side)
    side.synchronize()
    torch.cuda._sleep(LONG)
    late = out.clone()                   # still to come when `out` is freed
    del out, lse
    T.tree_verify_attention_shared(*other, **hint, stream=side)
    torch.cuda.synchronize()
    assert same([late], [want])
