"""GPU parity of the shared-prefix attention on values that its parts of rows have to
carry: infinities and NaN beside finite columns, in any part of a row."""
import numpy as np
import pytest
import torch

from tests import cache_util as C
from tests import gpu_util as U
from tests.test_gpu_cache import attend

pytestmark = pytest.mark.gpu

INF, NEG_INF, NAN = 0x7F80, 0xFF80, 0x7FC0


def special(w, b, t):
    page, slot = w.page_table[b, t // w.P], t % w.P
    for col, bits in ((7, INF), (9, NEG_INF), (11, NAN)):
        w.v_cache[page, slot, 1, col] = bits


def check_special(out):
    """+inf, -inf and NaN in their columns of KV head 1, nothing like them elsewhere."""
    got = U.bf16_to_f64(out) if isinstance(out, torch.Tensor) else out.copy()
    assert np.isposinf(got[..., 4:8, 7]).all() and np.isneginf(got[..., 4:8, 9]).all()
    assert np.isnan(got[..., 4:8, 11]).all()
    got[..., 4:8, [7, 9, 11]] = 0
    assert np.isfinite(got).all()


@pytest.mark.parametrize("N,D", [(2, 128), (12, 64), (24, 128), (64, 128), (100, 64)])
@pytest.mark.parametrize("length", [1, 9, 65, 73])
def test_an_infinity_ahead_of_missing_keys_stays_one(length, N, D):
    """The last cached row is the first of a load block: keys behind it are masked."""
    T = U.require_gpu()
    w = C.shared_workload(1010, B=1, N=N, Hq=8, Hkv=2, D=D, P=16, start=[0, 1], shared=[0], own=(length, length),
                          tree="chain", poison=False)
    special(w, 0, length - 1)
    check_special(attend(T, w, None, None)[0])
    check_special(U.gpu_attention(T, w)[0])


def test_an_infinity_ahead_of_missing_keys_of_own_row_blocks_stays_one():
    """The same behind shared row blocks (96 rows a sequence, 16 shared tiles)."""
    T = U.require_gpu()
    w = C.shared_workload(1011, B=6, N=24, Hq=8, Hkv=2, D=128, P=16, start=[0, 6], shared=[1024], own=(105, 105),
                          poison=False)
    special(w, 4, int(w.kv_len[4]) - 1)
    out, _ = attend(T, w, [0, 6], [1024], far=True)
    check_special(out[4])
    assert np.isfinite(U.bf16_to_f64(out)[[0, 1, 2, 3, 5]]).all()


@pytest.mark.parametrize("N,D", [(2, 128), (12, 64), (40, 128)])
@pytest.mark.parametrize("length", [200, 330, 390, 450, 520, 580, 777, 900, 1100, 1500, 2300])
def test_an_infinity_in_the_last_piece_stays_one(length, N, D):
    """Units split into two to twenty pieces, the last of which holds the last cached row."""
    T = U.require_gpu()
    w = C.shared_workload(1020, B=1, N=N, Hq=8, Hkv=2, D=D, P=16, start=[0, 1], shared=[0], own=(length, length),
                          tree="chain", poison=False)
    special(w, 0, length - 1)
    check_special(attend(T, w, None, None)[0])
