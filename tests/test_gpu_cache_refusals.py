"""Calls of the cache operators that are refused on the GPU machine only: the checks come behind
the one of the device."""
import numpy as np
import pytest
import torch

from tests import cache_util as C
from tests import gpu_util as U
from tests.test_gpu_cache import evict, upload_state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["kv_len", "seen", "fixed_len"])
@pytest.mark.parametrize("at", [-2, -1, 1, 2])
def test_kept_lengths_over_an_input_are_refused(name, at):
    """A view that shares some of the input's elements; beside them it is accepted."""
    T = U.require_gpu()
    from paper_2602_21224_amd._lib import TreeVerifyError
    s = C.cache_state(970, B=3, Hkv=2, D=64, P=16, lens=[100, 64, 40], fixed=4)
    d = upload_state(s)
    room = torch.full((12,), -5, dtype=torch.int32, device="cuda")
    room[4:7] = d[name]
    d[name] = room[4:7]
    before = [d[k].clone() for k in ("weight", "position", "k_cache", "v_cache")]
    with pytest.raises(TreeVerifyError, match="status -8 .*overlaps"):
        evict(T, s, d, 48, 8, kept_len=room[4 + at:7 + at])
    torch.cuda.synchronize()
    assert all(torch.equal(a.view(torch.int16), d[k].view(torch.int16))
               for a, k in zip(before, ("weight", "position", "k_cache", "v_cache")))
    assert (room[:4] == -5).all() and (room[7:] == -5).all()
    kept = evict(T, s, d, 48, 8, kept_len=room[7:10])[2]
    assert np.array_equal(kept.cpu().numpy(), [48, 48, 40])


@pytest.mark.parametrize("big", [(1 << 31) - 1, 1 << 31, 1 << 32, 1 << 40, (1 << 40) + 30])
def test_sizes_beyond_the_c_int_are_as_large_as_they_say(big):
    """Integers of which ctypes would pass the low 32 bits: 0 or 30 of the last three."""
    T = U.require_gpu()
    s = C.cache_state(971, B=3, Hkv=2, D=64, P=16, lens=[100, 64, 40], fixed=4)
    d = upload_state(s)
    kept = evict(T, s, d, big, 8, hint=big)[2]                 # no budget: nothing is evicted
    assert np.array_equal(kept.cpu().numpy(), s["kv_len"])
    assert np.array_equal(d["position"].cpu().numpy(), s["position"])
    want, got = upload_state(s), upload_state(s)
    a = evict(T, s, want, 48, 200)                             # all slots are recent ones
    b = evict(T, s, got, 48, big, hint=big)
    assert all(torch.equal(x.view(torch.int32), y.view(torch.int32)) for x, y in zip(a, b))


@pytest.mark.parametrize("low", [-1, -(1 << 31), -(1 << 32) + 48])
def test_negative_sizes_are_refused(low):
    T = U.require_gpu()
    from paper_2602_21224_amd._lib import TreeVerifyError
    s = C.cache_state(972, B=1, Hkv=2, D=64, P=16, lens=[64])
    d = upload_state(s)
    for kw in (dict(budget=low, recent=0), dict(budget=8, recent=low), dict(budget=8, recent=0, hint=low)):
        with pytest.raises(TreeVerifyError, match="status -2"):
            evict(T, s, d, **kw)
