"""GPU parity of the shared-prefix attention on values that its parts of rows have to
carry: infinities and NaN beside finite columns, in any part of a row."""
import numpy as np
import pytest
import torch

from paper_2602_21224_amd import workloads as W
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


def check_beside(oracle_mod, w, out, seqs, label):
    """`w` without the three special values, which KV head 1 of the sequences `seqs` has in
    columns 7, 9 and 11. Every other column is what it is without them: the attention's
    bound, and half a subnormal step of the fp16 parts, 2^-25 where a row's largest
    magnitude is 2^14 at least."""
    want, _, bound = C.attention_bounds(oracle_mod, w)
    mag = 2.0 ** 8 * bound                         # at least 2 sum p |v|
    bound = bound + 2.0 ** -39 * mag.max(-1, keepdims=True)
    got = U.bf16_to_f64(out)
    G = w.Hq // w.Hkv
    hit = np.zeros(got.shape[:3], bool)
    hit[seqs, :, G:2 * G] = True
    assert np.isposinf(got[hit][:, 7]).all() and np.isneginf(got[hit][:, 9]).all(), label
    assert np.isnan(got[hit][:, 11]).all(), label
    finite = np.ones(got.shape, bool)
    finite[np.ix_(seqs, range(w.N), range(G, 2 * G), (7, 9, 11))] = False
    err = np.where(finite, np.abs(np.where(finite, got, 0) - want), 0)
    print(f"[{label}] of its bound {(err / bound).max():.2f}", flush=True)
    assert (err <= bound).all(), label


def scale_values(w, power):
    f = np.float32(2.0 ** power)                   # exact: bf16 times a power of two
    w.v_cache = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.v_cache) * f)
    w.v_tree = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.v_tree) * f)


BESIDE = [
    # B, N, Hq, Hkv, D, P, shared, own, far
    (4, 2, 8, 2, 128, 16, 256, (10, 200), True),       # own units of 16 rows
    (3, 12, 8, 2, 64, 1, 320, (70, 400), True),        # of 48 rows, one-token pages
    (6, 24, 8, 2, 128, 16, 1024, (100, 300), True),    # shared and own row blocks
    (4, 2, 8, 2, 128, 16, 256, (10, 200), False),      # split units of 16 rows, nothing shared
    (4, 30, 8, 2, 64, 16, 256, (10, 200), False),      # of 128 rows
    (2, 64, 8, 2, 128, 16, 512, (300, 700), False),    # of 256 rows
]


@pytest.mark.parametrize("power", [0, 100, -100])
@pytest.mark.parametrize("case", range(len(BESIDE)))
def test_columns_beside_an_infinity_keep_their_values(oracle_mod, case, power):
    """+inf, -inf and NaN in a shared row, which every sequence sees, and in the last of
    one sequence's own rows."""
    T = U.require_gpu()
    B, N, Hq, Hkv, D, P, shared, own, far = BESIDE[case]
    w = C.shared_workload(1000 + case, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P, start=[0, B], shared=[shared], own=own,
                          tree="capped", poison=False)
    scale_values(w, power)
    clean = w.v_cache.copy()
    for where, b, t, seqs in (("shared", 0, 3, list(range(B))), ("own", 1, int(w.kv_len[1]) - 1, [1])):
        w.v_cache = clean.copy()
        special(w, b, t)
        out, _ = attend(T, w, [0, B], [shared], far=far)
        w.v_cache = clean
        check_beside(oracle_mod, w, out, seqs, f"beside{case} 2^{power} {where}")


@pytest.mark.parametrize("case", range(len(BESIDE)))
def test_parts_of_rows_keep_eleven_bits(case):
    """Queries of zeros weigh every key by exactly 1, so nothing is rounded but the parts
    and the output, whose true values are means of values 1 + k 2^-7 < 1.125: half a step
    of the output, 2^-8; half a step of the parts, whose weights' sum is 1, 2^-11 of them in
    fp16; fp32 sums, half a step 2^-24 a key, and some for the joining. Parts in bf16 (half a
    step 2^-8) put one value in 6 to 2000 outside this bound."""
    T = U.require_gpu()
    B, N, Hq, Hkv, D, P, shared, own, far = BESIDE[case]
    w = C.shared_workload(1040 + case, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P, start=[0, B], shared=[shared], own=own,
                          tree="chain", poison=False)
    rng = np.random.default_rng(case)
    for name in ("v_cache", "v_tree"):
        values = rng.integers(0, 16, getattr(w, name).shape).astype(np.float32) / 128 + 1
        setattr(w, name, W.f32_to_bf16_bits(values))
    w.q[:] = 0
    out, lse = attend(T, w, [0, B], [shared], far=far)
    got, z = U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64)
    tree = np.cumsum(W.bf16_bits_to_f32(w.v_tree).astype(np.float64), 1)       # a chain: node i sees 0 .. i
    worst = 0.0
    for b, L in enumerate(w.kv_len):
        t = np.arange(L)
        cached = W.bf16_bits_to_f32(w.v_cache[w.page_table[b, t // P], t % P]).astype(np.float64).sum(0)
        n = L + 1.0 + np.arange(N)
        mean = ((cached + tree[b]) / n[:, None, None]).repeat(Hq // Hkv, 1)
        bound = 2.0 ** -8 + 1.125 * (2.0 ** -11 + (L + N + 64) * 2.0 ** -24)
        worst = max(worst, np.abs(got[b] - mean).max() / bound)
        # log n, of sums of up to n ones and powers of 2
        assert (np.abs(z[b] - np.log(n)[:, None]) <= 2.0 ** -24 * (L + N + 64)).all()
    print(f"[parts{case}] of the bound {worst:.2f}", flush=True)
    assert worst <= 1
