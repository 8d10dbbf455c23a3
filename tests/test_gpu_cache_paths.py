"""GPU parity of the shared-prefix attention where keys are taken by groups: which path a
case runs is asserted from the rules, so that a changed rule cannot empty it."""
import numpy as np
import pytest
import torch

from tests import cache_util as C
from tests import gpu_util as U
from tests import shared_plan
from tests.test_gpu_cache import attend, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,grouped", [(1 << 20, True), (1 << 21, False)])
def test_page_tables_of_many_tokens(oracle_mod, tokens, grouped):
    """512 sequences x 32 KV heads with room for a million tokens each; of two million the
    places of own units are no longer counted and the batch takes the plain launch."""
    T = U.require_gpu()
    w = C.shared_workload(1100, B=512, N=1, Hq=32, Hkv=32, D=64, P=16, start=[0, 512], shared=[64], own=(0, 16),
                          tree="chain")
    assert shared_plan.by_groups(512, 1, 32, 32, 64, 1, tokens, tokens) == grouped
    d = U.upload(w)
    more = torch.full((512, tokens // 16 - w.page_table.shape[1]), -1, dtype=torch.int32, device="cuda")
    d["page_table"] = torch.cat([d["page_table"], more], 1)
    out, lse = T.tree_verify_attention_shared(
        d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"], d["page_table"], d["kv_len"], d["parent"],
        U.dev(np.array([0, 512], np.int32)), U.dev(np.array([64], np.int32)), max_kv_len=tokens)
    check_attention(oracle_mod, w, out, lse, f"{tokens} tokens")
