"""GPU parity of the cache operators against the CPU oracle: attention over
shared prefixes, accumulated weights, eviction, and a run of them together."""
import numpy as np
import pytest
import torch

from paper_2602_21224_amd import workloads as W
from tests import cache_util as C
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# attention over shared prefixes
# ---------------------------------------------------------------------------

def attend(T, w, start, shared, d=None, far=False, **kw):
    """far: the page table has columns and the bound allows lengths at which keys are
    taken by groups; without, these small batches are taken as if nothing were shared."""
    d = d or U.upload(w)
    if far:
        d = {**d, "page_table": far_table(w, d["page_table"])}
    i32 = lambda a: a if a is None or isinstance(a, torch.Tensor) else U.dev(np.asarray(a, np.int32))  # noqa: E731
    return T.tree_verify_attention_shared(
        d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"], d["page_table"], d["kv_len"], d["parent"],
        i32(start), i32(shared), max_kv_len=1 << 24 if far else w.max_kv_len, num_nodes=d["num_nodes"], **kw)


def far_table(w, table):
    tokens = -(-(256 << 20) // (w.B * w.Hkv * w.D * 4))
    more = torch.full((w.B, max(1, -(-tokens // w.P) - table.shape[1])), -1, dtype=torch.int32, device="cuda")
    return torch.cat([table, more], 1)


def check_attention(oracle_mod, w, out, lse, label):
    got, z = U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64)
    want, zw, bound = C.attention_bounds(oracle_mod, w)
    nodes = np.full(w.B, w.N) if w.num_nodes is None else w.num_nodes
    real = np.arange(w.N)[None, :] < nodes[:, None]
    assert (got[~real] == 0).all() and np.isneginf(z[~real]).all(), label
    err = np.abs(got - want)[real]
    print(f"[{label}] max abs err {err.max(initial=0):.2e}, "
          f"of its bound {(err / bound[real]).max(initial=0):.2f}", flush=True)
    assert np.isfinite(got[real]).all() and (err <= bound[real]).all(), label
    norm = lambda x: np.sqrt(np.nanmax((W.bf16_bits_to_f32(x) ** 2).sum(-1), initial=0))  # noqa: E731
    qk = norm(w.q) * max(norm(w.k_tree), norm(w.k_cache)) / np.sqrt(w.D)
    tol = C.lse_bound(w.D, qk) + 2.0 ** -21 * np.abs(zw[real])
    assert (np.abs(z - zw)[real] <= tol).all(), (label, np.abs(z - zw)[real].max())


SHARED = [
    # B, N, Hq, Hkv, D, P, start, shared, own, ragged, tree
    (4, 1, 8, 2, 128, 16, [0, 4], [256], (0, 70), False, "chain"),           # decoding
    (64, 1, 32, 8, 128, 16, [0, 64], [512], (0, 200), False, "chain"),       # a large decoding batch
    (3, 12, 8, 8, 64, 16, [0, 3], [128], (0, 0), False, "capped"),           # nothing but the shared tokens
    (5, 45, 24, 8, 64, 1, [0, 2, 5], [300, 129], (0, 90), True, "forest"),   # two groups, odd sizes, one-token pages
    (6, 16, 12, 4, 128, 8, [1, 4], [200], (1, 150), True, "capped"),         # sequences outside every group
    (4, 64, 32, 8, 128, 16, [0, 4], [1024], (0, 400), False, "capped"),      # 1024 rows of a group per KV head
    (3, 100, 16, 2, 64, 64, [0, 3], [640], (0, 130), True, "capped"),        # G = 8, several row blocks
    (2, 256, 8, 8, 128, 16, [0, 2], [192], (1, 300), False, "chain"),        # the largest trees
    (7, 5, 6, 2, 128, 2, [0, 2, 2, 4, 7], [64, 0, 0, 130], (0, 40), True, "forest"),   # an empty group, a length of 0
    (3, 7, 5, 1, 64, 256, [0, 3], [1280], (0, 600), False, "forest"),        # pages longer than a tile
    (2, 3, 4, 4, 128, 16, [0, 2], [32], (0, 20), False, "forest"),           # shared lengths below a tile
    (8, 24, 8, 1, 128, 4, [0, 8], [1500], (0, 64), True, "capped"),          # one KV head
    (6, 24, 16, 4, 128, 16, [0, 4, 6], [512, 192], (0, 150), False, "capped"),   # 96 rows: blocks of several sequences
    (5, 16, 4, 2, 64, 16, [0, 5], [960], (100, 900), True, "forest"),        # 32 rows, long own parts
    (9, 3, 32, 2, 128, 1, [0, 9], [333], (1, 70), False, "chain"),           # 48 rows, one-token pages
    (5, 100, 6, 2, 128, 16, [0, 2, 5], [1600, 256], (0, 200), True, "capped"),   # 300 rows, two blocks
    (4, 140, 4, 1, 64, 16, [0, 4], [2048], (0, 300), False, "forest"),       # 560 rows, three blocks
]


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("case", range(len(SHARED)))
def test_shared_attention(oracle_mod, case, far):
    T = U.require_gpu()
    B, N, Hq, Hkv, D, P, start, shared, own, ragged, tree = SHARED[case]
    w = C.shared_workload(700 + case, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P, start=start, shared=shared, own=own,
                          ragged=ragged, tree=tree)
    print(f"case shared{case}: {SHARED[case]} nodes={w.num_nodes}", flush=True)
    out, lse = attend(T, w, start, shared, far=far)
    check_attention(oracle_mod, w, out, lse, f"shared{case} {far}")
    again, lse2 = attend(T, w, start, shared, far=far)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("start,shared", [
    (None, None),                        # no groups
    ([0, 3], [0]),
    ([0, 3], [63]), ([0, 3], [100]), ([0, 3], [129]),   # less than what is shared, odd
    ([0, 3], [1 << 30]),                 # more than any sequence has: cut to the shortest
    ([0, 1, 2, 3], [192, 192, 192]),     # groups of one
    ([0, 2, 1, 3], [192, 192, 192]),     # not ascending: counts as 0, 2, 2, 3
    ([-5, 9], [192]),                    # outside [0, B]: clamped
    ([1, 3], [-4]),
])
def test_shared_lengths_and_groups_change_nothing(oracle_mod, start, shared, far):
    """Whatever is promised of the sharing (as far as it is true), the function is the
    attention's."""
    T = U.require_gpu()
    w = C.shared_workload(720, B=3, N=9, Hq=8, Hkv=2, D=128, P=16, start=[0, 3], shared=[192], own=(0, 90))
    if shared is not None and max(shared) > 192:
        w.kv_len[:] = [192, 150, 192]
        w.k_cache[w.k_cache == W.BF16_NAN] = 0
        w.v_cache[w.v_cache == W.BF16_NAN] = 0
    out, lse = attend(T, w, start, shared, far=far)
    check_attention(oracle_mod, w, out, lse, f"{start} {shared}")


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("power", [100, -100])
@pytest.mark.parametrize("N", [2, 30])
def test_parts_of_any_magnitude_are_joined(oracle_mod, power, N, far):
    """Values far outside fp16's range, and a row with an infinity: what is left of the
    two parts in the workspace is scaled per row."""
    T = U.require_gpu()
    w = C.shared_workload(745, B=4, N=N, Hq=8, Hkv=2, D=128, P=16, start=[0, 4], shared=[256], own=(10, 200),
                          tree="chain", poison=False)
    f = np.float32(2.0 ** power)
    # no rounding: a bf16 times a power of two
    w.v_cache = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.v_cache) * f)
    w.v_tree = W.f32_to_bf16_bits(W.bf16_bits_to_f32(w.v_tree) * f)
    out, lse = attend(T, w, [0, 4], [256], far=far)
    check_attention(oracle_mod, w, out, lse, f"2^{power}")
    w.v_cache[w.page_table[0, 0], 3, 1, 7] = 0x7F80              # an infinity that every row of KV head 1 sees
    inf, _ = attend(T, w, [0, 4], [256], far=far)
    a, b = U.bf16_to_f64(inf), U.bf16_to_f64(out)
    hit = np.zeros(a.shape, bool)
    hit[:, :, 4:, 7] = True
    assert np.isposinf(a[hit]).all() and np.isfinite(a[~hit]).all()
    assert np.array_equal(a[:, :, :4], b[:, :, :4])
    if power == 100:
        # an infinite row's parts are scaled by 2^-113: fp16 steps of 2^-24 there, for each of two parts,
        # and the output's own rounding on both sides
        np.testing.assert_allclose(a[~hit], b[~hit], rtol=2.0 ** -7, atol=2.0 * 2.0 ** (113 - 24))


@pytest.mark.parametrize("far", [False, True])
def test_the_largest_batch_of_groups(oracle_mod, far):
    """512 sequences in 256 groups of any length, some of them empty."""
    T = U.require_gpu()
    rng = np.random.default_rng(8)
    start = np.sort(np.append(rng.integers(0, 513, 255), [0, 512]))
    shared = (rng.integers(0, 20, 256) * 16).tolist()
    w = C.shared_workload(746, B=512, N=2, Hq=3, Hkv=1, D=64, P=16, start=start, shared=shared, own=(0, 40),
                          tree="forest")
    out, lse = attend(T, w, start, shared, far=far)
    check_attention(oracle_mod, w, out, lse, "256 groups")


@pytest.mark.parametrize("far", [False, True])
def test_shared_attention_of_empty_sequences(oracle_mod, far):
    """A group whose first sequence has no nodes (its length and pages hold anything),
    and one where none has."""
    T = U.require_gpu()
    w = C.shared_workload(730, B=5, N=10, Hq=8, Hkv=2, D=64, P=16, start=[0, 3, 5], shared=[128, 64],
                          own=(0, 40), ragged=True)
    w.num_nodes[:] = [0, 7, 10, 0, 0]
    rng = np.random.default_rng(1)
    w.parent[1, :7] = W.tree_uniform_forest(rng, 7)
    w.parent[2, :10] = W.tree_uniform_forest(rng, 10)
    fill = lambda x: np.where(x == W.BF16_NAN, np.uint16(0x3F80), x)  # noqa: E731
    w.q, w.k_tree, w.v_tree = fill(w.q), fill(w.k_tree), fill(w.v_tree)
    ref = W.Workload(**{**w.__dict__, "page_table": w.page_table.copy(), "kv_len": w.kv_len.copy()})
    w.page_table[0], w.page_table[3] = -9, 1 << 30
    w.kv_len[0], w.kv_len[3] = 3, -2
    out, lse = attend(T, w, [0, 3, 5], [128, 64], far=far)
    check_attention(oracle_mod, ref, out, lse, "empty")


def test_shared_attention_equals_the_plain_one_without_groups():
    T = U.require_gpu()
    w = C.shared_workload(731, B=3, N=20, Hq=8, Hkv=2, D=128, P=16, start=[0, 3], shared=[256], own=(5, 90))
    a, za = attend(T, w, None, None)
    b, zb = U.gpu_attention(T, w)
    assert np.abs(U.bf16_to_f64(a) - b).max() <= 2.0 ** -6 and np.abs(za.cpu().numpy() - zb).max() <= 1e-4


@pytest.mark.parametrize("far", [False, True])
def test_shared_attention_needs_no_lse_and_no_clean_workspace(oracle_mod, far):
    T = U.require_gpu()
    w = C.shared_workload(732, B=4, N=12, Hq=8, Hkv=8, D=128, P=16, start=[0, 4], shared=[320], own=(0, 200))
    out, lse = attend(T, w, [0, 4], [320], far=far)
    need = T.shared_attention_workspace_size(w.B, w.N, w.Hq, w.Hkv, w.D, 1)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    again, none = attend(T, w, [0, 4], [320], far=far, workspace=ws, want_lse=False)
    assert none is None and torch.equal(out.view(torch.int16), again.view(torch.int16))


# ---------------------------------------------------------------------------
# accumulated weights
# ---------------------------------------------------------------------------

def upload_state(s):
    bits = ("k_cache", "v_cache", "q")
    return {k: (U.dev_bf16(v) if k in bits else U.dev(v)) for k, v in s.items()}


def weight_case(seed, *, B, N, Hq, Hkv, D, P, lens, path, fixed):
    rng = np.random.default_rng(seed)
    s = C.cache_state(seed, B=B, Hkv=Hkv, D=D, P=P, lens=lens, room=N, fixed=fixed, poison=False)
    idx, alen = C.accepted_paths(rng, B, N, path)
    # slots past the path hold NaN: they are not read into any sum
    W.poison_cache_tails(s["k_cache"], s["v_cache"], s["page_table"], s["kv_len"] + alen, P)
    q = W.f32_to_bf16_bits(rng.standard_normal((B, N, Hq, D), dtype=np.float32))
    lse = (np.log(np.asarray(lens) + 1.0)[:, None, None] + 0.5 + 0.1 * rng.standard_normal((B, N, Hq)))
    lse = lse.astype(np.float32)
    rest = np.ones((B, N), bool)         # nodes that were not accepted: never read
    for b in range(B):
        rest[b, idx[b, :alen[b]]] = False
    q[rest], lse[rest] = W.BF16_NAN, np.nan
    return dict(s, q=q, lse=lse, accept_idx=idx, accept_len=alen)


def accumulate(T, s, d, **kw):
    return T.kv_accumulate_weights(d["q"], d["lse"], d["k_cache"], d["page_table"], d["kv_len"], d["accept_idx"],
                                   d["accept_len"], d["weight"], d["position"], d["seen"],
                                   max_kv_len=kw.pop("hint", int(s["kv_len"].max(initial=0))),
                                   fixed_len=kw.pop("fixed_len", d["fixed_len"]), **kw)


def check_weights(oracle_mod, s, weight, position, label, scale=0.0, fixed="fixed_len", before=None):
    names = ("q", "lse", "k_cache", "page_table", "kv_len", "accept_idx", "accept_len", "weight", "position",
             "seen")
    want, pos = oracle_mod.accumulate_weights(*(s[n] for n in names), fixed_len=s[fixed] if fixed else None,
                                              scale=scale)
    got = weight.cpu().numpy().astype(np.float64)
    if before is not None:               # a buffer of its own: what lies past the path stays as it was
        T = got.shape[2]
        past = np.arange(T) >= (s["kv_len"] + s["accept_len"])[:, None, None]
        want = np.where(past, before, want)
    assert np.array_equal(position.cpu().numpy(), pos), label
    # each exponential's argument is off by the dot product's fp32 sums (half a step 2^-24
    # of sum |q_i k_i| <= |q||k| per addition) and some steps of its terms; the sums of
    # positive terms by half a step per addition, for every row and the old weight
    D, G = s["q"].shape[3], s["q"].shape[2] // s["k_cache"].shape[2]
    norm = lambda x: np.sqrt(np.nanmax((W.bf16_bits_to_f32(x) ** 2).sum(-1), initial=0))  # noqa: E731
    qk = norm(s["q"]) * norm(s["k_cache"]) * (scale or D ** -0.5)
    z = np.nanmax(np.abs(np.where(np.isfinite(s["lse"]), s["lse"], 0)), initial=0)
    rel = 2.0 ** -24 * ((D + 8) * qk + 4 * (qk + z) + G * s["accept_len"].max(initial=0) + 8)
    err = np.abs(got - want)
    print(f"[{label}] max rel err {(err / np.maximum(np.abs(want), 1e-30)).max():.2e}, bound {rel:.2e}", flush=True)
    assert (err <= rel * np.abs(want) + 1e-37).all(), label


WEIGHTS = [
    # B, N, Hq, Hkv, D, P, lens, path lengths, fixed
    (1, 1, 8, 8, 64, 16, [128], [1], 0),
    (3, 1, 8, 2, 128, 16, [0, 1, 65], [1, 1, 0], 0),               # nothing cached yet; nothing accepted
    (4, 16, 32, 8, 128, 16, [17, 64, 300, 1000], [1, 4, 16, 9], 16),
    (2, 45, 24, 8, 64, 1, [301, 77], [45, 20], 7),                 # 135 rows, three heads, one-token pages
    (2, 33, 14, 2, 128, 8, [63, 129], [33, 32], 0),                # seven heads
    (1, 256, 16, 2, 64, 64, [500], [256], 100),                    # 2048 rows
    (2, 12, 5, 1, 128, 256, [900, 255], [3, 12], 64),              # a page that ends inside a tile
    (2, 8, 4, 4, 128, 2, [40, 90], [2, 5], 1000),                  # everything fixed
    (5, 6, 8, 2, 64, 4, [7, 2049, 100, 0, 31], [6, 1, 3, 2, 5], 3),
    (2, 16, 8, 8, 128, 16, [48, 112], [16, 16], 40),               # the last slot of the table is taken
]


@pytest.mark.parametrize("case", range(len(WEIGHTS)))
def test_accumulated_weights(oracle_mod, case):
    T = U.require_gpu()
    B, N, Hq, Hkv, D, P, lens, path, fixed = WEIGHTS[case]
    s = weight_case(800 + case, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P, lens=lens, path=path, fixed=fixed)
    print(f"case weights{case}: {WEIGHTS[case]}", flush=True)
    d = upload_state(s)
    before = torch.full_like(d["weight"], 7.5)
    position = d["position"].clone()
    w, p = accumulate(T, s, {**d, "position": position}, weight_out=before.clone())
    check_weights(oracle_mod, s, w, p, f"weights{case}", before=7.5)
    assert torch.equal(d["weight"].cpu(), torch.from_numpy(s["weight"]))
    w2, p2 = accumulate(T, s, d, hint=1)                           # in place, and a bound that is far too low
    assert w2 is d["weight"] and p2 is d["position"]
    end = (s["kv_len"] + s["accept_len"])[:, None, None] > np.arange(w.shape[2])
    assert torch.equal(w2[U.dev(np.broadcast_to(end, w.shape))], w[U.dev(np.broadcast_to(end, w.shape))])
    check_weights(oracle_mod, s, w2, p2, f"weights{case} in place")


def test_accumulated_weights_without_fixed_slots_and_with_a_scale(oracle_mod):
    T = U.require_gpu()
    s = weight_case(820, B=2, N=6, Hq=8, Hkv=2, D=64, P=16, lens=[90, 200], path=[6, 2], fixed=0)
    d = upload_state(s)
    w, p = accumulate(T, s, d, fixed_len=None, scale=0.3, weight_out=torch.zeros_like(d["weight"]))
    check_weights(oracle_mod, s, w, p, "scale", scale=0.3, fixed=None, before=0.0)


def test_rows_that_saw_nothing_add_nothing(oracle_mod):
    """lse -inf, node ids out of range, page ids out of range."""
    T = U.require_gpu()
    s = weight_case(821, B=2, N=6, Hq=8, Hkv=2, D=64, P=16, lens=[90, 200], path=[4, 6], fixed=0)
    s["lse"][0, s["accept_idx"][0, 1], 3] = -np.inf
    s["lse"][1, s["accept_idx"][1, 0]] = -np.inf
    d = upload_state(s)
    w, p = accumulate(T, s, d, weight_out=torch.zeros_like(d["weight"]))
    check_weights(oracle_mod, s, w, p, "lse", before=0.0)
    bad = s["accept_idx"].copy()
    lse = s["lse"].copy()
    lse[1, bad[1, 5]] = -np.inf          # what a skipped row comes to
    bad[1, 5] = 6
    table = s["page_table"].copy()
    table[0, 2] = 1 << 20
    wb, _ = accumulate(T, s, {**d, "accept_idx": U.dev(bad), "page_table": U.dev(table)},
                       weight_out=torch.full_like(d["weight"], -3.0))
    ref, _ = accumulate(T, s, {**d, "lse": U.dev(lse)}, weight_out=torch.full_like(d["weight"], -3.0))
    ref[0, :, 32:48] = -3.0
    assert torch.equal(wb, ref)


def test_weights_of_a_real_attention_sum_to_one():
    """With the lse of the attention over the same keys every row gives away one."""
    T = U.require_gpu()
    w = C.shared_workload(822, B=3, N=8, Hq=16, Hkv=4, D=128, P=16, start=[0, 3], shared=[128], own=(0, 300),
                          tree="chain")
    d = U.upload(w)
    _, lse = attend(T, w, [0, 3], [128], d)
    alen = U.dev(np.array([8, 1, 5], np.int32))
    idx = U.dev(np.where(np.arange(8) < np.array([8, 1, 5])[:, None], np.arange(8), -1).astype(np.int32))
    T.kv_compact_accepted(d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"], d["page_table"], d["kv_len"], idx,
                          alen)
    slots = (3, 4, w.page_table.shape[1] * 16)
    weight, _ = T.kv_accumulate_weights(d["q"], lse, d["k_cache"], d["page_table"], d["kv_len"], idx, alen,
                                        torch.zeros(slots, device="cuda"),
                                        torch.zeros(slots, dtype=torch.int32, device="cuda"), d["kv_len"],
                                        max_kv_len=w.max_kv_len)
    want = alen[:, None].float() * 4
    # the lse is off by its bound, about 2e-4 here, and the sums by some 2^-24 a term
    assert ((weight.sum(-1) - want).abs() <= 4e-4 * want).all()


# ---------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------

def evict(T, s, d, budget, recent, **kw):
    return T.kv_evict(d["weight"], d["position"], d["k_cache"], d["v_cache"], d["page_table"], d["kv_len"],
                      d["seen"], max_kv_len=kw.pop("hint", int(s["kv_len"].max(initial=0))), budget=budget,
                      recent=recent, fixed_len=kw.pop("fixed_len", d["fixed_len"]), **kw)


def check_evict(oracle_mod, s, got, k, v, budget, recent, label, before=None, fixed="fixed_len"):
    w, p, kc, vc, kept = oracle_mod.evict(*(s[n] for n in ("weight", "position", "k_cache", "v_cache",
                                                           "page_table", "kv_len", "seen")),
                                          budget=budget, recent=recent, fixed_len=s[fixed] if fixed else None)
    if before is not None:
        past = np.arange(w.shape[2]) >= kept[:, None, None]
        w, p = np.where(past, before[0], w), np.where(past, before[1], p)
    gw, gp, gl = (t.cpu().numpy() for t in got)
    assert np.array_equal(gl, kept), label
    assert np.array_equal(gp, p), label
    np.testing.assert_array_equal(gw.view(np.int32), w.astype(np.float32).view(np.int32), err_msg=label)
    assert np.array_equal(k.view(torch.int16).cpu().numpy().view(np.uint16), kc), label
    assert np.array_equal(v.view(torch.int16).cpu().numpy().view(np.uint16), vc), label


EVICT = [
    # B, Hkv, D, P, lens, budget, recent, fixed, ties
    (1, 8, 64, 16, [128], 96, 16, 4, False),
    (4, 2, 128, 16, [0, 1, 33, 300], 32, 8, 2, False),             # empty, one slot, one too many
    (3, 3, 64, 1, [501, 40, 77], 41, 10, 0, True),                 # one-token pages, many equal weights
    (2, 4, 128, 8, [900, 1024], 100, 200, 30, True),               # the recent ones alone exceed the budget
    (2, 2, 128, 256, [700, 300], 512, 0, 0, False),
    (3, 2, 8, 4, [100, 64, 20], 10, 3, 50, True),                  # more fixed than the budget
    (2, 1, 1024, 16, [2500, 1025], 1024, 1, 1, False),             # more slots than threads, wide rows
    (2, 2, 64, 16, [200, 90], 0, 5, 0, False),                     # nothing may stay
    (1, 2, 64, 16, [20000], 15000, 500, 64, False),
    (1, 1, 64, 32, [40000], 9001, 7, 0, True),
    (2, 2, 72, 16, [100, 70], 60, 0, 3, False),                    # a head size of no other operator
]


@pytest.mark.parametrize("case", range(len(EVICT)))
def test_eviction(oracle_mod, case):
    T = U.require_gpu()
    B, Hkv, D, P, lens, budget, recent, fixed, ties = EVICT[case]
    s = C.cache_state(900 + case, B=B, Hkv=Hkv, D=D, P=P, lens=lens, fixed=fixed, ties=ties)
    print(f"case evict{case}: {EVICT[case]}", flush=True)
    d = upload_state(s)
    k, v = d["k_cache"].clone(), d["v_cache"].clone()
    wo, po = torch.full_like(d["weight"], -1.5), torch.full_like(d["position"], -99)
    got = evict(T, s, {**d, "k_cache": k, "v_cache": v}, budget, recent, weight_out=wo, position_out=po)
    check_evict(oracle_mod, s, got, k, v, budget, recent, f"evict{case}", before=(-1.5, -99))
    got = evict(T, s, d, budget, recent, hint=1)                   # in place, and a bound that is far too low
    assert got[0] is d["weight"] and got[1] is d["position"]
    check_evict(oracle_mod, s, got, d["k_cache"], d["v_cache"], budget, recent, f"evict{case} in place")


def test_eviction_orders_special_weights_as_the_argmax_does(oracle_mod):
    """NaN stays before infinity, -0 ties with 0, -inf and the lowest finite value go first."""
    T = U.require_gpu()
    s = C.cache_state(930, B=1, Hkv=4, D=64, P=16, lens=[64])
    rng = np.random.default_rng(3)
    pool = np.array([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, np.finfo(np.float32).min, -1.0, 1e-45, -1e-45],
                    np.float32)
    s["weight"][:] = rng.choice(pool, s["weight"].shape)
    for budget in (1, 13, 31, 40, 50, 63):
        d = upload_state(s)
        got = evict(T, s, d, budget, 0, fixed_len=None)
        check_evict(oracle_mod, s, got, d["k_cache"], d["v_cache"], budget, 0, f"special {budget}", fixed=None)


def test_eviction_of_extreme_positions(oracle_mod):
    T = U.require_gpu()
    s = C.cache_state(931, B=2, Hkv=2, D=64, P=16, lens=[64, 50])
    top = np.iinfo(np.int32)
    s["position"][0, :, ::3] = top.max
    s["position"][1, :, ::2] = top.min
    s["seen"][:] = [top.max, top.min]
    for recent in (0, 1, top.max):
        d = upload_state(s)
        got = evict(T, s, d, 30, recent)
        check_evict(oracle_mod, s, got, d["k_cache"], d["v_cache"], 30, recent, f"recent {recent}")


def test_rows_of_pages_out_of_range_stay(oracle_mod):
    """Nothing outside the pool is read or written; the other rows move as they would."""
    T = U.require_gpu()
    s = C.cache_state(932, B=2, Hkv=2, D=64, P=16, lens=[128, 100])
    d = upload_state(s)
    table = s["page_table"].copy()
    table[0, 1], table[1, 4] = -1, table.max() + 1
    k, v = d["k_cache"].clone(), d["v_cache"].clone()
    got = evict(T, s, {**d, "k_cache": k, "v_cache": v, "page_table": U.dev(table)}, 64, 0,
                weight_out=torch.zeros_like(d["weight"]), position_out=torch.zeros_like(d["position"]))
    w, p, kc, vc, kept = oracle_mod.evict(s["weight"], s["position"], s["k_cache"], s["v_cache"],
                                          s["page_table"], s["kv_len"], s["seen"], 64, 0, s["fixed_len"])
    assert np.array_equal(got[2].cpu().numpy(), kept)
    assert np.array_equal(got[1].cpu().numpy()[:, :, :64], p[:, :, :64])
    a = k.view(torch.int16).cpu().numpy().view(np.uint16)
    old = {int(x): i for i, x in enumerate(s["position"][1, 0, :100])}
    for t in range(64):
        i = old[int(p[1, 0, t])]
        to = (s["page_table"][1, t // 16], t % 16, 0)
        want = s["k_cache"][to] if i // 16 == 4 else kc[to]
        np.testing.assert_array_equal(a[to], want)
    assert (a[s["page_table"][0, 1]] == s["k_cache"][s["page_table"][0, 1]]).all()


# ---------------------------------------------------------------------------
# streams, graphs, and a loop of them all
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("far", [False, True])
def test_calls_on_other_streams(far):
    """Two calls at once, each on its own stream with its own workspace."""
    T = U.require_gpu()
    w = C.shared_workload(940, B=4, N=16, Hq=16, Hkv=4, D=128, P=16, start=[0, 4], shared=[512], own=(0, 300))
    s = C.cache_state(941, B=3, Hkv=4, D=64, P=16, lens=[900, 700, 40])
    d, e = U.upload(w), upload_state(s)
    want, wz = attend(T, w, [0, 4], [512], d, far)
    copy = lambda: {**e, "k_cache": e["k_cache"].clone(), "v_cache": e["v_cache"].clone(),  # noqa: E731
                    "weight": e["weight"].clone(), "position": e["position"].clone()}
    ref = copy()
    kept = evict(T, s, ref, 256, 30)
    two = [copy(), copy()]
    # inputs live until the other streams are done with them
    start, shared = U.dev(np.array([0, 4], np.int32)), U.dev(np.array([512], np.int32))
    d["page_table"] = far_table(w, d["page_table"]) if far else d["page_table"]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    hint = 1 << 24 if far else w.max_kv_len
    outs = [T.tree_verify_attention_shared(d["q"], d["k_tree"], d["v_tree"], d["k_cache"], d["v_cache"],
                                           d["page_table"], d["kv_len"], d["parent"], start, shared,
                                           max_kv_len=hint, num_nodes=d["num_nodes"], stream=st) for st in streams]
    kepts = [evict(T, s, x, 256, 30, stream=st) for x, st in zip(two, streams)]
    torch.cuda.synchronize()
    for (o, z), x, k in zip(outs, two, kepts):
        assert torch.equal(o.view(torch.int16), want.view(torch.int16)) and torch.equal(z, wz)
        assert all(torch.equal(a, b) for a, b in zip(k, kept))
        assert torch.equal(x["k_cache"].view(torch.int16), ref["k_cache"].view(torch.int16))


@pytest.mark.parametrize("far", [False, True])
def test_a_captured_step_replays(far):
    """Attention, weights and eviction in one graph, replayed on new inputs with eager
    work between the replays."""
    T = U.require_gpu()
    w = C.shared_workload(950, B=3, N=8, Hq=8, Hkv=2, D=128, P=16, start=[0, 3], shared=[192], own=(0, 120),
                          tree="chain", poison=False)
    d = U.upload(w)
    at, hint = (far_table(w, d["page_table"]), 1 << 24) if far else (d["page_table"], w.max_kv_len)
    slots = (3, 2, w.page_table.shape[1] * 16)
    gs, sl = U.dev(np.array([0, 3], np.int32)), U.dev(np.array([192], np.int32))
    alen, idx = U.dev(np.array([3, 1, 8], np.int32)), torch.arange(8, dtype=torch.int32, device="cuda").repeat(3, 1)
    weight, position = torch.zeros(slots, device="cuda"), torch.zeros(slots, dtype=torch.int32, device="cuda")
    w1, w2, p2 = torch.empty_like(weight), torch.empty_like(weight), torch.empty_like(position)
    out, lse = torch.empty_like(d["q"]), torch.empty((3, 8, 8), device="cuda")
    kept = torch.empty(3, dtype=torch.int32, device="cuda")
    ws = torch.empty(T.shared_attention_workspace_size(3, 8, 8, 2, 128, 1), dtype=torch.uint8, device="cuda")
    we = torch.empty(T.evict_workspace_size(3, 2, w.page_table.shape[1], 16), dtype=torch.uint8, device="cuda")
    kc, vc = d["k_cache"].clone(), d["v_cache"].clone()
    fixed = torch.full((3,), 192, dtype=torch.int32, device="cuda")   # shared pages: no row of them may move

    def step():
        kc.copy_(d["k_cache"])
        vc.copy_(d["v_cache"])
        w1.zero_(), w2.zero_(), p2.zero_()
        T.tree_verify_attention_shared(d["q"], d["k_tree"], d["v_tree"], kc, vc, at, d["kv_len"],
                                       d["parent"], gs, sl, max_kv_len=hint, out=out, lse=lse, workspace=ws)
        T.kv_compact_accepted(d["k_tree"], d["v_tree"], kc, vc, d["page_table"], d["kv_len"], idx, alen)
        T.kv_accumulate_weights(d["q"], lse, kc, d["page_table"], d["kv_len"], idx, alen, weight, position,
                                d["kv_len"], max_kv_len=w.max_kv_len, weight_out=w1)
        end = d["kv_len"] + alen
        T.kv_evict(w1, position, kc, vc, d["page_table"], end, end, max_kv_len=w.max_kv_len + 8, budget=230,
                   recent=16, fixed_len=fixed, weight_out=w2, position_out=p2, kept_len=kept, workspace=we)

    def seen():
        torch.cuda.synchronize()
        return [t.clone() for t in (out.view(torch.int16), lse, kc.view(torch.int16), vc.view(torch.int16), w1, w2,
                                    p2, kept)]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(k)
        d["q"].copy_(torch.randn(d["q"].shape, generator=gen, device="cuda"))
        weight.copy_(torch.rand(slots, generator=gen, device="cuda"))
        graph.replay()
        got = seen()
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, seen())), k


@pytest.mark.parametrize("far", [False, True])
def test_a_serving_loop_with_a_shared_prompt_and_a_budget(oracle_mod, far):
    """Several steps of verification over one cache: attention over the shared prompt,
    acceptance, compaction, weights, eviction of what each sequence has of its own,
    against the oracle run on the same states."""
    T = U.require_gpu()
    B, N, Hq, Hkv, D, P, prompt, budget = 3, 10, 8, 2, 64, 16, 64, 90
    rng = np.random.default_rng(960)
    lens = np.array([70, 88, 64], np.int32)
    per = -(-(budget + 4 * N) // P) + 1
    table = rng.permutation(B * per).astype(np.int32).reshape(B, per)
    table[1:, :prompt // P] = table[0, :prompt // P]
    bits = lambda *s: W.f32_to_bf16_bits(rng.standard_normal(s, dtype=np.float32))  # noqa: E731
    kc, vc = bits(B * per, P, Hkv, D), bits(B * per, P, Hkv, D)
    seen = lens.copy()
    slots = (B, Hkv, per * P)
    position = np.broadcast_to(np.arange(per * P, dtype=np.int32), slots).copy()
    weight = np.zeros(slots, np.float32)
    fixed = np.full(B, prompt, np.int32)
    dk, dv, dw, dp = U.dev_bf16(kc), U.dev_bf16(vc), U.dev(weight), U.dev(position)
    dt, df = U.dev(table), U.dev(fixed)
    gs, sl = U.dev(np.array([0, B], np.int32)), U.dev(np.array([prompt], np.int32))
    evicted = 0
    for step in range(6):
        q, kt, vt = bits(B, N, Hq, D), bits(B, N, Hkv, D), bits(B, N, Hkv, D)
        parent = np.stack([W.tree_chain(N)] * B)
        draft = rng.integers(0, 9, (B, N)).astype(np.int32)
        logits = rng.standard_normal((B, N, 9), dtype=np.float32)
        for b in range(B):               # the next node's token wins with probability 0.8
            for i in range(N - 1):
                if rng.random() < 0.8:
                    logits[b, i, draft[b, i + 1]] += 20
        dl, ds, dpar = U.dev(lens), U.dev(seen), U.dev(parent)
        gq, gk, gv = U.dev_bf16(q), U.dev_bf16(kt), U.dev_bf16(vt)
        w = W.Workload("loop", B, N, Hq, Hkv, D, P, 9, q, kt, vt, kc, vc, table, lens, parent, draft, None)
        at, hint = (far_table(w, dt), 1 << 24) if far else (dt, int(lens.max()))
        out, lse = T.tree_verify_attention_shared(gq, gk, gv, dk, dv, at, dl, dpar, gs, sl, max_kv_len=hint)
        _, alen, idx, _ = T.tree_argmax_accept(U.dev(logits), U.dev(draft), dpar)
        T.kv_compact_accepted(gk, gv, dk, dv, dt, dl, idx, alen)
        T.kv_accumulate_weights(gq, lse, dk, dt, dl, idx, alen, dw, dp, ds, max_kv_len=int(lens.max()), fixed_len=df)
        dl, ds = dl + alen, ds + alen
        top = int(dl.max())
        w_in = dw.cpu().numpy()          # the oracle evicts by the weights that the kernels summed
        *_, kept = T.kv_evict(dw, dp, dk, dv, dt, dl, ds, max_kv_len=top, budget=budget, recent=8, fixed_len=df)
        torch.cuda.synchronize()

        check_attention(oracle_mod, w, out, lse, f"step {step}")
        al, ai = alen.cpu().numpy(), idx.cpu().numpy()
        kc, vc = oracle_mod.kv_compact(kt, vt, kc, vc, table, lens, ai, al)
        state = dict(q=q, lse=lse.cpu().numpy(), k_cache=kc, page_table=table, kv_len=lens, accept_idx=ai,
                     accept_len=al, weight=weight, position=position, seen=seen, fixed_len=fixed)
        _, position = oracle_mod.accumulate_weights(**state)
        check_weights(oracle_mod, state, torch.from_numpy(w_in), torch.from_numpy(position), f"step {step}")
        lens, seen = lens + al, seen + al
        evicted += int((lens > budget).sum())
        weight, position, kc, vc, lens = oracle_mod.evict(w_in, position, kc, vc, table, lens, seen, budget, 8, fixed)
        weight = weight.astype(np.float32)
        assert np.array_equal(kept.cpu().numpy(), lens)
        assert np.array_equal(dp.cpu().numpy(), position) and np.array_equal(dw.cpu().numpy(), weight)
        assert np.array_equal(dk.view(torch.int16).cpu().numpy().view(np.uint16), kc)
        assert np.array_equal(dv.view(torch.int16).cpu().numpy().view(np.uint16), vc)
    assert evicted >= 5 and lens.max() <= budget
