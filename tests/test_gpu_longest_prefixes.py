"""Attention over prefixes whose positions reach the end of the int32 range. Windows hold a
few resident pages of them; calls without a window read the same pages again and again."""
import numpy as np
import pytest
import torch

from paper_2602_21224_amd import workloads as W
from tests import cache_util as C
from tests import gpu_util as U
from tests import long_util as LU

pytestmark = pytest.mark.gpu

LONGEST = 0x7FFFFFFF - 1024


@pytest.mark.parametrize("which", ["window", "4 bits"])
@pytest.mark.parametrize("N", [1, 40])
@pytest.mark.parametrize("D,P,back", [(64, 4, 0), (64, 4, 2000), (128, 16, 0), (128, 16, 8000), (128, 256, 0),
                                      (128, 256, 100000), (128, 256, 200001)])
def test_a_window_at_the_end_of_the_longest_table(which, N, D, P, back):
    """As a short prefix whose pages before the window are gone: positions count only by
    their distance."""
    T = U.require_gpu()
    window, sinks = 1024, 70
    columns = LONGEST // P
    L = columns * P - back
    gone = (L - 3000) // P                                     # pages that the short prefix lacks
    w = LU.workload(71, B=1, N=N, Hq=8, Hkv=2, D=D, P=P, lens=[L - gone * P], window=window, sinks=sinks)
    print(f"{which} N {N} D {D} P {P}: {L} tokens, {L - gone * P} held", flush=True)
    d = U.upload(w)
    first = -(-sinks // P)
    held = d["page_table"][:, :-(-(L - gone * P) // P)]
    table = torch.full((1, columns), -1, dtype=torch.int32, device="cuda")
    table[:, :first] = held[:, :first]
    table[:, gone + first:gone + held.shape[1]] = held[:, first:]
    bits = None if which == "window" else LU.cache4(w)
    cache = [d["k_cache"], d["v_cache"]] if bits is None else [U.dev(a) for a in bits]
    f = T.tree_verify_attention_window if bits is None else T.tree_verify_attention_kv4
    out, lse = f(d["q"], d["k_tree"], d["v_tree"], *cache, table, torch.tensor([L], dtype=torch.int32, device="cuda"),
                 d["parent"], max_kv_len=L, window=window, sinks=sinks)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, window, sinks, bits),
             f"{which} {N} {P} {back}")


@pytest.mark.parametrize("N", [1, 40])
@pytest.mark.parametrize("P,columns", [(256, 1 << 23), (256, (1 << 24) + 3), (16, 1 << 27)])
def test_a_table_with_room_for_more_tokens_than_a_prefix_can_have(N, P, columns):
    T = U.require_gpu()
    w = LU.workload(72, B=1, N=N, Hq=8, Hkv=2, D=128, P=P, lens=[777])
    print(f"N {N} P {P} columns {columns}", flush=True)
    d = U.upload(w)
    table = torch.full((1, columns), -1, dtype=torch.int32, device="cuda")
    table[:, :w.page_table.shape[1]] = d["page_table"]
    out, lse = T.tree_verify_attention(d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"], table, d["kv_len"],
                                       d["parent"], max_kv_len=777)
    want, z = U.gpu_attention(T, w, d=d)
    assert np.array_equal(U.bf16_to_f64(out), want) and np.array_equal(lse.cpu().numpy(), z)


@pytest.mark.parametrize("window,sinks", [(0, 0), (600, 5)])
@pytest.mark.parametrize("N,Hq,L", [(12, 96, 300), (12, 96, 2500), (40, 48, 2500), (1, 24, 700)])
def test_4_bits_in_a_table_for_more_row_blocks_than_are_counted(N, Hq, L, window, sinks):
    """24 KV heads in a table of nearly 2^31 tokens: blocks of 32 rows would be too many tiles."""
    T = U.require_gpu()
    w = LU.workload(73, B=1, N=N, Hq=Hq, Hkv=24, D=64, P=256, lens=[L], window=window, sinks=sinks)
    print(f"N {N} Hq {Hq} L {L} window {window}", flush=True)
    d, bits = U.upload(w), LU.cache4(w)
    table = torch.full((1, LONGEST // 256), -1, dtype=torch.int32, device="cuda")
    table[:, :w.page_table.shape[1]] = d["page_table"]
    out, lse = T.tree_verify_attention_kv4(d["q"], d["k_tree"], d["v_tree"], *[U.dev(a) for a in bits], table, d["kv_len"],
                                           d["parent"], max_kv_len=L, window=window, sinks=sinks)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, window, sinks, bits),
             f"{N} {Hq} {L} {window}")


@pytest.mark.parametrize("shared", [False, True])
def test_a_prefix_of_nearly_2_to_the_31_tokens(shared):
    """All pages but the last 390 are one page of zeros (weight 1 each); those hold keys of
    weights around e^25, which all have to be there."""
    T = U.require_gpu()
    B, D, P, ends = 3 if shared else 1, 64, 256, 390
    columns = LONGEST // P
    L = columns * P - 1234
    rng = np.random.default_rng(5)
    bits = lambda *s: W.f32_to_bf16_bits(rng.standard_normal(s, dtype=np.float32))  # noqa: E731
    q, k_tree, v_tree = bits(1, 1, 1, D), bits(1, 1, 1, D), bits(1, 1, 1, D)
    k, v = bits(ends + 1, P, 1, D), bits(ends + 1, P, 1, D)
    qf = W.bf16_bits_to_f32(q)[0, 0, 0].astype(np.float64)
    kf = W.bf16_bits_to_f32(k).astype(np.float64)
    # moved along q so that the scores' mean is 25
    k = W.f32_to_bf16_bits((kf + qf * (25 * np.sqrt(D) / (qf @ qf))).astype(np.float32))
    k[ends], v[ends] = 0, 0
    last = L - (columns - ends) * P                            # keys of the last pages
    kt = W.bf16_bits_to_f32(k)[:ends, :, 0].reshape(-1, D)[:last].astype(np.float64)
    vt = W.bf16_bits_to_f32(v)[:ends, :, 0].reshape(-1, D)[:last].astype(np.float64)
    kt = np.concatenate([kt, W.bf16_bits_to_f32(k_tree)[0, :, 0]])
    vt = np.concatenate([vt, W.bf16_bits_to_f32(v_tree)[0, :, 0]])
    weight = np.exp(kt @ qf / np.sqrt(D))
    total = weight.sum() + (columns - ends) * P
    want, mag, z = weight @ vt / total, weight @ np.abs(vt) / total, np.log(total)

    up = lambda a: U.dev_bf16(np.repeat(a, B, axis=0))  # noqa: E731
    table = torch.full((B, columns), ends, dtype=torch.int32, device="cuda")
    table[:, columns - ends:] = torch.arange(ends, dtype=torch.int32, device="cuda")
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    args = (up(q), up(k_tree), up(v_tree), U.dev_bf16(k), U.dev_bf16(v), table, lens,
            torch.full((B, 1), -1, dtype=torch.int32, device="cuda"))
    print(f"shared {shared}: {L} tokens", flush=True)
    if shared:
        out, lse = T.tree_verify_attention_shared(*args, torch.tensor([0, B], dtype=torch.int32, device="cuda"),
                                                  torch.tensor([L], dtype=torch.int32, device="cuda"), max_kv_len=L)
    else:
        out, lse = T.tree_verify_attention(*args, max_kv_len=L)
    # weights, a split row's part and the output rounded to bf16 (half a step 2^-8, of the
    # weights, the part and the output), scores and fp32 exponentials as elsewhere, and fp32
    # sums of the last pages' tiles: two additions each, half a step 2^-24 of the sum so far
    qk = np.sqrt(qf @ qf) * np.sqrt((kt ** 2).sum(-1).max()) / np.sqrt(D)
    sums = 2 * (last / 64 + 2) * 2.0 ** -24
    ztol = C.lse_bound(D, qk) + sums + 2.0 ** -21 * z
    tol = 2.0 ** -8 * (2 * mag + np.abs(want)) + (2.0 ** -12 + 2 * ztol + sums) * mag
    got, zg = U.bf16_to_f64(out)[:, 0, 0], lse.cpu().numpy().astype(np.float64)[:, 0, 0]
    err, zerr = np.abs(got - want), np.abs(zg - z)
    print(f"of the bound {(err / tol).max():.2f}, lse {(zerr / ztol).max():.2f} ({zerr.max():.1e})", flush=True)
    assert (err <= tol).all() and (zerr <= ztol).all()
