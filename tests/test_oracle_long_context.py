"""Pins of the long-context oracle (CPU only): the 4-bit form against its definition value
by value, and the window against the plain attention."""
import numpy as np
import pytest

from oracle import long_context as O
from paper_2602_21224_amd import workloads as W
from tests import long_util as LU


def bits(x):
    return W.f32_to_bf16_bits(np.asarray(x, np.float32))


def row(values, fill=0.0):
    x = np.full(32, fill, np.float32)
    x[:len(values)] = values
    return bits(x)


def test_codes_of_known_values():
    # a 4 in the block fixes e = 0: every midpoint goes to the even code
    c, e = O.quantize4(row([4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, 6, -6, 0.0, -0.0, 0.2, 0.3]))
    n = np.stack([c & 15, c >> 4], -1).reshape(-1)
    assert e.tolist() == [127]
    assert n[:16].tolist() == [6, 0, 2, 2, 4, 4, 6, 6, 8, 10, 7, 15, 0, 8, 0, 1]


@pytest.mark.parametrize("top,e", [(6.0, 0), (7.0, 0), (7.03125, 1), (8.0, 1), (3.5, -1), (3.515625, 0), (1.0, -2),
                                   (2.0 ** -130, -126), (0.0, -126), (1.4 * 2.0 ** 127, 125), (3.3895e38, 125)])
def test_the_smallest_power_of_two_with_which_the_largest_is_at_most_seven(top, e):
    _, byte = O.quantize4(row([top, -top / 3]))
    assert int(byte[0]) - 127 == e


def test_blocks_that_four_bits_cannot_hold_are_nan_whole():
    x = np.ones((3, 64), np.float32)
    x[0, 5], x[1, 40], x[2, 63] = np.nan, np.inf, -np.inf
    c, e = O.quantize4(bits(x))
    assert (e == 255).tolist() == [[True, False], [False, True], [False, True]]
    y = O.dequantize4(c, e)
    assert np.isnan(y[0, :32]).all() and (y[0, 32:] == 1).all() and np.isnan(y[1, 32:]).all()
    assert (c[0, :16] == 0).all()


def test_values_come_back_exactly_and_within_half_a_step():
    rng = np.random.default_rng(0)
    x = bits(rng.standard_normal((50, 128)) * np.exp2(rng.integers(-90, 90, size=(50, 1))))
    c, e = O.quantize4(x)
    y = O.dequantize4(c, e)
    v = W.bf16_bits_to_f32(x).astype(np.float64)
    power = np.repeat(2.0 ** (e.astype(np.float64) - 127), 32, axis=-1)
    assert (np.abs(y - v) <= power * np.where(np.abs(v) / power > 4, 1.0, np.where(np.abs(v) / power > 2, 0.5, 0.25))).all()
    again = O.quantize4(bits(y))                 # exact in bf16, and its own nearest value
    assert np.array_equal(O.dequantize4(*again), y)
    assert np.array_equal(W.bf16_bits_to_f32(bits(y)).astype(np.float64), y)


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 9), (4096, 0), (400, 3)])
def test_a_window_over_everything_is_the_plain_attention(oracle_mod, window, sinks):
    w = LU.workload(3, B=3, N=9, Hq=6, Hkv=2, D=64, P=4, lens=[0, 37, 300], tree="forest")
    out, lse, _ = O.window_attention(w.q, w.k_tree, w.v_tree, O.Rows16(w.k_cache), O.Rows16(w.v_cache), w.page_table,
                                     w.kv_len, w.parent, window, sinks)
    want, zw = oracle_mod.tree_attention(w.q, w.k_tree, w.v_tree, w.k_cache, w.v_cache, w.page_table, w.kv_len, w.parent)
    np.testing.assert_allclose(out, want, rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(lse, zw, rtol=1e-10, atol=1e-12)


def test_a_chain_in_a_window_is_causal_attention_with_a_band():
    """Position by position: the chain's nodes are the sequence's last tokens."""
    w = LU.workload(4, B=1, N=11, Hq=2, Hkv=1, D=64, P=4, lens=[20], tree="chain")
    out, _, _ = O.window_attention(w.q, w.k_tree, w.v_tree, O.Rows16(w.k_cache), O.Rows16(w.v_cache), w.page_table,
                                   w.kv_len, w.parent, 6, 2)
    t = np.arange(20)
    k = np.concatenate([W.bf16_bits_to_f32(w.k_cache)[w.page_table[0, t // 4], t % 4, 0],
                        W.bf16_bits_to_f32(w.k_tree)[0, :, 0]]).astype(np.float64)
    v = np.concatenate([W.bf16_bits_to_f32(w.v_cache)[w.page_table[0, t // 4], t % 4, 0],
                        W.bf16_bits_to_f32(w.v_tree)[0, :, 0]]).astype(np.float64)
    at = np.arange(31)
    band = (at[None, :] <= at[20:, None]) & ((at[None, :] < 2) | (at[None, :] > at[20:, None] - 6))
    assert band.sum(1).tolist() == [8] * 11
    s = W.bf16_bits_to_f32(w.q)[0, :, 1].astype(np.float64) @ k.T / 8
    p = np.where(band, np.exp(s), 0)
    np.testing.assert_allclose(out[0, :, 1], (p / p.sum(1, keepdims=True)) @ v, rtol=1e-10, atol=1e-12)


def test_a_window_of_one_leaves_the_node_itself_and_the_sinks():
    w = LU.workload(5, B=1, N=5, Hq=1, Hkv=1, D=64, P=4, lens=[9], tree="chain")
    for sinks, first in ((0, []), (2, [0, 1])):
        rows = O.visible(w.parent[0], 9, 5, 1, sinks)
        assert all(pos.tolist() == first and path == [i] for i, (pos, path) in enumerate(rows))
    # sinks that reach into the tree: the first path nodes stay visible
    rows = O.visible(w.parent[0], 9, 5, 1, 11)
    assert rows[4][0].tolist() == list(range(9)) and rows[4][1] == [0, 1, 4]


def test_write_goes_through_table_index_and_count():
    rng = np.random.default_rng(1)
    k, v = bits(rng.standard_normal((2, 3, 2, 64))), bits(rng.standard_normal((2, 3, 2, 64)))
    zero = lambda *s: np.zeros(s, np.uint8)  # noqa: E731
    table = np.array([[5, 1], [0, 3]], np.int32)
    k4, v4, sc, hk, hv = O.write4(k, v, zero(6, 2, 2, 32), zero(6, 2, 2, 32), zero(6, 2, 2, 2, 2), table, [1, 0],
                                  idx=np.array([[2, 0, -1], [1, 1, 1]]), count=[2, 1])
    assert np.array_equal(O.dequantize4(k4[5, :, 1], sc[5, :, 1, 0]), hk[0, 0])
    assert np.array_equal(O.dequantize4(v4[1, :, 0], sc[1, :, 0, 1]), hv[0, 1])
    assert np.array_equal(hk[1, 0], O.dequantize4(*O.quantize4(k[1, 1]))) and (hk[1, 1:] == 0).all()
    touched = (sc != 0).any(axis=(1, 3, 4))
    assert np.argwhere(touched).tolist() == [[0, 0], [1, 0], [5, 1]]
