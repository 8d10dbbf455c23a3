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
