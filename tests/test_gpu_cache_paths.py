"""GPU parity of the shared-prefix attention where keys are taken by groups: which path a
case runs is asserted from the rules, so that a changed rule cannot empty it."""
import numpy as np
import pytest
import torch

from tests import cache_util as C
from tests import gpu_util as U
from tests import shared_plan
from tests.test_gpu_cache import attend, check_attention, far_table

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


BY_GROUPS = [
    # B, N, Hq, Hkv, D, P, start, shared, own, ragged, tree, tiles taken together (None: some)
    # row blocks, the groups' and the sequences' own
    (6, 24, 8, 2, 128, 1, [0, 6], [1500], (0, 200), False, "capped", [23]),     # one-token pages: three page windows
    (6, 24, 8, 2, 64, 1, [0, 6], [1500], (0, 200), False, "forest", [23]),
    (9, 20, 12, 4, 64, 2, [0, 9], [1300], (0, 90), True, "forest", None),       # 60 rows at most, ragged
    (6, 100, 6, 2, 128, 1, [0, 3, 6], [1600, 640], (0, 700), False, "capped", [25, 0]),   # 300 rows, own windows too
    (5, 64, 6, 2, 128, 16, [0, 5], [2240], (0, 90), False, "chain", [35]),      # 192 rows
    (12, 12, 16, 2, 128, 4, [2, 12], [1024], (1, 150), True, "capped", None),   # sequences outside the group
    (4, 140, 4, 1, 64, 1, [0, 4], [2048], (0, 300), False, "forest", [32]),     # 560 rows, trees over 64 nodes
    (9, 100, 6, 2, 64, 1, [0, 9], [2048], (0, 300), True, "forest", None),      # the same, ragged
    (6, 24, 8, 2, 128, 256, [0, 6], [1280], (0, 600), False, "forest", [20]),   # pages longer than a tile
    (16, 24, 16, 4, 128, 16, [0, 8, 16], [2048, 1024], (0, 500), False, "capped", [32, 16]),   # units longer than shares
    (7, 75, 4, 2, 64, 8, [0, 7], [1500], (0, 90), False, "capped", [23]),       # 150 rows, the last tile not shared
    # units of 16, 32 and 48 rows that waves take by themselves, one-token pages past the page window
    (4, 3, 8, 2, 64, 1, [0, 4], [1500], (600, 900), False, "chain", [23]),
    (4, 8, 8, 2, 128, 1, [0, 4], [1500], (0, 900), False, "capped", [23]),
    (4, 8, 8, 2, 64, 1, [0, 4], [1500], (0, 90), True, "forest", None),
    (3, 12, 8, 2, 64, 2, [0, 3], [1700], (0, 300), False, "forest", [26]),
    (3, 12, 8, 2, 128, 1, [0, 3], [1700], (0, 300), False, "capped", [26]),
]


@pytest.mark.parametrize("case", range(len(BY_GROUPS)))
def test_keys_taken_by_groups(oracle_mod, case):
    T = U.require_gpu()
    B, N, Hq, Hkv, D, P, start, shared, own, ragged, tree, tiles = BY_GROUPS[case]
    w = C.shared_workload(1200 + case, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P, start=start,
                          shared=[n // P * P for n in shared], own=own, ragged=ragged, tree=tree)
    d = U.upload(w)
    tokens = far_table(w, d["page_table"]).shape[1] * P
    assert shared_plan.by_groups(B, N, Hq, Hkv, D, len(shared), min(tokens, 1 << 24), tokens)
    took = shared_plan.shared_tiles(w, start, shared)
    assert took == tiles if tiles is not None else max(took) > 0
    print(f"case by_groups{case}: {BY_GROUPS[case]} nodes={w.num_nodes}", flush=True)
    out, lse = attend(T, w, start, shared, d, far=True)
    check_attention(oracle_mod, w, out, lse, f"by_groups{case}")
    again, lse2 = attend(T, w, start, shared, d, far=True)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)
