"""Every value that 4 bits and a scale byte can stand for, through the attention over them:
subnormal ones as they are, infinite ones from 2^128 on, NaN."""
import numpy as np
import pytest

from oracle import long_context as O
from paper_2602_21224_amd import workloads as W
from tests import gpu_util as U
from tests import long_util as LU

pytestmark = pytest.mark.gpu

SHAPES = [(1, 64, 1), (1, 128, 16), (40, 128, 2), (80, 64, 16), (200, 128, 1)]      # by waves, by workgroups


def attend(T, w, cache):
    d = U.upload(w)
    out, lse = T.tree_verify_attention_kv4(d["q"], d["k_tree"], d["v_tree"], *[U.dev(a) for a in cache], d["page_table"],
                                           d["kv_len"], d["parent"], max_kv_len=1)
    return U.bf16_to_f64(out)[:, :, 0], lse.cpu().numpy().astype(np.float64)[:, :, 0]


def one_key_per_byte(N, D, P):
    """Sequence b has one cached key, in slot 0 of a page."""
    w = LU.workload(39, B=256, N=N, Hq=1, Hkv=1, D=D, P=P, lens=[1] * 256, tree="forest")
    w.parent[:] = -1
    w.k_tree[:], w.v_tree[:] = 0, 0
    return w, LU.cache4(w), w.page_table[:, 0]


@pytest.mark.parametrize("N,D,P", SHAPES)
def test_every_scale_byte_and_code_of_v(N, D, P):
    """The node itself has weight e^-48, whose V is 0, so out is the cached row."""
    T = U.require_gpu()
    print(f"N {N} D {D} P {P}", flush=True)
    w, (k4, v4, sc), pages = one_key_per_byte(N, D, P)
    w.q[:] = W.f32_to_bf16_bits(np.array([3.0], np.float32))[0]
    k4[pages, 0, 0], sc[pages] = 0x44, 127                     # 2 everywhere: scores 48 and 67.9
    v4[pages, 0, 0] = [(2 * i % 16) + 16 * ((2 * i + 1) % 16) for i in range(D // 2)]
    sc[pages, 0, 0, 1] = np.arange(256)[:, None]
    got, _ = attend(T, w, (k4, v4, sc))
    want = O.dequantize4(v4[pages, 0, 0], sc[pages, 0, 0, 1])
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.isinf(want).sum() == 6 * D // 8 and np.isnan(want[255]).all() and np.isfinite(want[:253]).all()
    for i in range(N):
        assert np.array_equal(got[:, i], want, equal_nan=True), i


@pytest.mark.parametrize("N,D,P", SHAPES)
def test_every_scale_byte_of_k(N, D, P):
    """One column of the cached key is not 0, and q there a power of two that brings the
    score near 1; the node's own score is 0."""
    T = U.require_gpu()
    print(f"N {N} D {D} P {P}", flush=True)
    w, (k4, v4, sc), pages = one_key_per_byte(N, D, P)
    byte = np.arange(256)
    power = np.clip(127.0 - byte, -126, 127)
    k4[pages, 0, 0], v4[pages, 0, 0], sc[pages] = 0, 0, 127
    sc[pages, 0, 0, 0] = byte[:, None]
    code, at = byte % 7 + 1, 32 * (byte // 7 % (D // 32)) + byte % 32
    k4[pages, 0, 0, at // 2] = code << 4 * (at % 2)
    w.q[:] = 0
    w.q[byte, :, 0, at] = W.f32_to_bf16_bits((2.0 ** power).astype(np.float32))[:, None]
    got, lse = attend(T, w, (k4, v4, sc))
    score = O.GRID[code] * 2.0 ** (byte - 127 + power) / np.sqrt(D)
    ok = byte < 253                                            # from 2^128 on K is infinite, and 255 is NaN
    assert (score[ok] >= 0.5 / 16).all() and (score[ok] <= 6).all()
    # fp32: the score's scale and exponential, the sum and its logarithm, a step (2^-23) each
    # of values up to 8
    want = np.log1p(np.exp(score))
    assert (np.abs(lse - want[:, None])[ok] <= 4 * 8 * 2.0 ** -23).all()
    assert (got[ok] == 0).all() and np.isnan(lse[255]).all()
