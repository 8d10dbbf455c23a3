"""Scores that are NaN reach out and lse of the rows that have them, and nothing else, however
a row's keys are divided: the plain attention and the one over shared prefixes."""
import pytest
import torch

from tests import gpu_util as U
from tests import long_util as LU

pytestmark = pytest.mark.gpu


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def check(run, k_cache, pages, rows, heads, seen):
    """NaN in KV head 0 of the K rows `rows` of `pages`, seen by the sequences `seen`."""
    out, lse = run()
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    keep = k_cache.clone()
    k_cache[pages, rows, 0] = float("nan")
    bad, z = run()
    k_cache.copy_(keep)
    hit = torch.zeros(lse.shape, dtype=torch.bool, device="cuda")
    hit[seen, :, :heads] = True
    assert torch.isnan(bad[hit]).all() and torch.isnan(z[hit]).all()
    assert same(bad[~hit], out[~hit]) and torch.equal(z[~hit], lse[~hit])


@pytest.mark.parametrize("D,P", [(64, 16), (128, 4), (128, 1)])
@pytest.mark.parametrize("B,N", [(1, 1), (1, 64), (700, 1), (300, 9), (200, 64)])
def test_plain(B, N, D, P):
    T = U.require_gpu()
    print(f"B {B} N {N} D {D} P {P}", flush=True)
    w = LU.workload(37, B=B, N=N, Hq=8, Hkv=2, D=D, P=P, lens=[1500] + [70] * (B - 1), tree="forest")
    d = U.upload(w)

    def run():
        return T.tree_verify_attention(d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"], d["page_table"],
                                       d["kv_len"], d["parent"], max_kv_len=1500)
    for first, last in ((64, 320), (128, 129)):                # whole tiles, and one key
        t = torch.arange(first, last, device="cuda")
        check(run, d["k_cache"], d["page_table"][0, t // P].long(), t % P, 4, [0])


@pytest.mark.parametrize("groups", [0, 1])
@pytest.mark.parametrize("N", [1, 14, 40, 64])
@pytest.mark.parametrize("D,P", [(64, 2), (128, 16)])
def test_shared(N, D, P, groups):
    T = U.require_gpu()
    B, Hkv, L, shared = 10, 8, 4096 + 700, 4096
    print(f"N {N} D {D} P {P} groups {groups}", flush=True)
    w = LU.workload(38, B=B, N=N, Hq=Hkv, Hkv=Hkv, D=D, P=P, lens=[L] * B, tree="forest")
    w.page_table[:, :shared // P] = w.page_table[0, :shared // P]
    d = U.upload(w)
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = (ints(0, B), ints(shared)) if groups else (None, None)

    def run():
        return T.tree_verify_attention_shared(d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"],
                                              d["page_table"], d["kv_len"], d["parent"], *plan, max_kv_len=L)
    for first, last, b, seen in ((640, 3008, 0, slice(0, B)), (4160, L, 3, [3]), (700, 701, 0, slice(0, B))):
        t = torch.arange(first, last, device="cuda")
        check(run, d["k_cache"], d["page_table"][b, t // P].long(), t % P, 1, seen)
