"""Cases of the cache operators: attention over shared prefixes, accumulated
attention weights, eviction by weight.

A serving loop whose requests begin with the same long prompt verifies their
draft trees with `tree_verify_attention_shared`, adds the attention that the
accepted tokens paid to each cached key with `kv_accumulate_weights`, and, when
a cache has grown past its budget, drops the keys that got least with
`kv_evict`. The listed cases take each call at the sizes of this repository's
presets and between them; the drawn ones spread over the same ranges.
Workspaces and output buffers are kept between calls, as a serving loop keeps
them. A pass leaves its inputs as they were (the updated weights and positions
go to buffers of their own; an eviction moves rows into slots that it reads
nothing from), so that the next one finds the same work.
"""
import math

import numpy as np
import torch

own = False

BF16 = torch.bfloat16


def listed():
    return [
        # Plain decoding (one token a sequence) of a batch behind one long system prompt.
        dict(name="shared_decode_b64", kind="shared", B=64, N=1, Hq=32, Hkv=8, D=128, P=16, groups=1,
             slo=4096, shi=4096, lo=16, hi=512, tree="chain", ragged=False),
        # Multi-head attention with the narrow 12-token trees that the method verifies.
        dict(name="shared_mha_b16", kind="shared", B=16, N=12, Hq=32, Hkv=32, D=128, P=16, groups=1,
             slo=1024, shi=1024, lo=0, hi=1024, tree="capped", ragged=False),
        # Small: forests of different sizes in two groups, head size 64, one-token pages,
        # three heads per KV head, odd lengths.
        dict(name="shared_ragged_d64", kind="shared", B=5, N=45, Hq=24, Hkv=8, D=64, P=1, groups=2,
             slo=300, shi=777, lo=0, hi=301, tree="forest", ragged=True),
        # Grouped-query attention of an 8B-shaped layer, 16 requests of two prompts.
        dict(name="shared_gqa_b16", kind="shared", B=16, N=64, Hq=32, Hkv=8, D=128, P=16, groups=2,
             slo=1024, shi=4096, lo=64, hi=1024, tree="capped", ragged=False),
        # The largest: a 70B-shaped layer behind a long document.
        dict(name="shared_gqa70_b16", kind="shared", B=16, N=64, Hq=64, Hkv=8, D=128, P=16, groups=1,
             slo=16384, shi=16384, lo=128, hi=1024, tree="capped", ragged=False),
        # One short sequence, one accepted token.
        dict(name="weights_tiny", kind="weights", B=1, N=1, Hq=8, Hkv=8, D=64, P=16, lo=128, hi=128,
             amax=1, fixed=0),
        # 8B-shaped, 16 requests, paths of up to 8 accepted tokens.
        dict(name="weights_gqa_b16", kind="weights", B=16, N=64, Hq=32, Hkv=8, D=128, P=16, lo=1024,
             hi=4096, amax=8, fixed=16),
        # Long accepted paths, three heads per KV head, one-token pages, odd lengths.
        dict(name="weights_long_path_d64", kind="weights", B=5, N=45, Hq=24, Hkv=8, D=64, P=1, lo=301,
             hi=2503, amax=45, fixed=7),
        # The longest prefixes.
        dict(name="weights_long_b4", kind="weights", B=4, N=256, Hq=32, Hkv=8, D=128, P=16, lo=32768,
             hi=32768, amax=12, fixed=64),
        # One short sequence that is a quarter over its budget.
        dict(name="evict_tiny", kind="evict", B=1, Hkv=8, D=64, P=16, lo=128, hi=128, budget=96,
             recent=16, fixed=4),
        # A batch in steady state, at most a few hundred tokens over the budget, some below it.
        dict(name="evict_gqa_b16", kind="evict", B=16, Hkv=8, D=128, P=16, lo=1900, hi=2311,
             budget=2048, recent=256, fixed=16),
        # Long prompts cut to a quarter at once.
        dict(name="evict_long_b4", kind="evict", B=4, Hkv=8, D=128, P=16, lo=32768, hi=32768,
             budget=8192, recent=1024, fixed=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    Hkv = rng.choice([2, 4, 8, 8, 16, 32])
    return Hkv, Hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])


def draw(rng):
    kind = rng.choice(["shared", "shared", "weights", "weights", "evict"])
    while True:
        Hkv, Hq = _heads(rng)
        D, P = rng.choice([64, 128, 128]), rng.choice([1, 2, 8, 16, 16, 16, 32, 64, 256])
        N = rng.choice([1, _log_int(rng, 2, 256)])
        if kind == "shared":
            B = _log_int(rng, 2, 96)
            shi, hi = _log_int(rng, 64, 16384), _log_int(rng, 1, 2048)
            c = dict(kind=kind, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P,
                     groups=rng.choice([1, 1, 2, max(1, B // 3)]), slo=rng.choice([shi, shi // 2]), shi=shi,
                     lo=rng.choice([hi, hi // 2, 0]), hi=hi, tree=rng.choice(["forest", "capped", "chain"]),
                     ragged=N >= 12 and rng.random() < 0.3)
            if N * Hq > 2048 * Hkv or work(c)["flops"] > 5e11 or B * (shi + hi) * Hkv * D > 4e8:
                continue
        elif kind == "weights":
            hi = _log_int(rng, 64, 32768)
            c = dict(kind=kind, B=_log_int(rng, 1, 64), N=N, Hq=Hq, Hkv=Hkv, D=D, P=P,
                     lo=rng.choice([hi, hi // 2, hi // 4]), hi=hi, amax=rng.choice([1, min(N, 8), min(N, 16), N]),
                     fixed=rng.choice([0, 4, hi // 8]))
            if N * Hq > 2048 * Hkv or work(c)["flops"] > 5e10 or c["B"] * hi * Hkv * D > 1.4e8:
                continue
        else:
            hi = _log_int(rng, 64, 32768)
            budget = max(8, int(hi * rng.choice([0.25, 0.5, 0.8, 0.95])))
            c = dict(kind=kind, B=_log_int(rng, 1, 64), Hkv=Hkv, D=D, P=P, lo=rng.choice([hi, hi // 2]), hi=hi,
                     budget=budget, recent=rng.choice([0, 1, budget // 8, budget // 2]),
                     fixed=rng.choice([0, 4, budget // 8]))
            if c["B"] * hi * Hkv * D > 1.4e8:
                continue
        return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _parents(rng, case):
    """Parent links [B, N] and node counts [B] (padding nodes: -1)."""
    B, N = case["B"], case["N"]
    parent = np.full((B, N), -1, dtype=np.int32)
    counts = np.full(B, N, dtype=np.int32)
    if case["ragged"]:
        counts = rng.integers(max(1, N // 3), N + 1, size=B).astype(np.int32)
    for i in range(1, N):
        if case["tree"] == "chain":
            parent[:, i] = i - 1
        elif case["tree"] == "forest":
            parent[:, i] = rng.integers(-1, i, size=B)
        else:                            # shallow: a parent among the first quarter of the nodes
            parent[:, i] = rng.integers(0, i // 4 + 1, size=B)
    parent[np.arange(N)[None, :] >= counts[:, None]] = -1
    return parent, counts


def _table(rng, case, room, shared=None, start=None):
    """Page table [B, max_pages] of random pages with `room` more tokens after the
    longest prefix; members of group s take its first shared[s] tokens' pages from its
    first."""
    B, P = case["B"], case["P"]
    per = -(-(case.get("shi", 0) + case["hi"] + room) // P)
    table = rng.permutation(B * per).astype(np.int32).reshape(B, per)
    if shared is not None:
        for s, n in enumerate(shared):
            table[start[s]:start[s + 1], :n // P] = table[start[s], :n // P]
    return table, B * per


def prepare(case, seed):
    B, Hkv, D, P = (case[k] for k in ("B", "Hkv", "D", "P"))
    rng, g = np.random.default_rng(seed), _gen(seed)
    bf = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=BF16)  # noqa: E731
    lens = rng.integers(case["lo"], case["hi"] + 1, size=B).astype(np.int32)
    s = dict(case=case)
    if case["kind"] == "shared":
        N, Hq, S = case["N"], case["Hq"], case["groups"]
        start = np.linspace(0, B, S + 1).astype(np.int32)
        shared = (rng.integers(case["slo"], case["shi"] + 1, size=S) // P * P).astype(np.int32)
        lens = lens + np.repeat(shared, np.diff(start)).astype(np.int32)
        table, pages = _table(rng, case, N, shared, start)
        parent, counts = _parents(rng, case)
        s.update(q=bf(B, N, Hq, D), k_tree=bf(B, N, Hkv, D), v_tree=bf(B, N, Hkv, D),
                 k_cache=bf(pages, P, Hkv, D), v_cache=bf(pages, P, Hkv, D), page_table=_dev(table),
                 kv_len=_dev(lens), parent=_dev(parent), group_start=_dev(start), shared_len=_dev(shared),
                 num_nodes=_dev(counts) if case["ragged"] else None, max_kv_len=int(lens.max()),
                 out=torch.empty((B, N, Hq, D), dtype=BF16, device="cuda"),
                 lse=torch.empty((B, N, Hq), dtype=torch.float32, device="cuda"), workspace=None)
        return s
    room = case["N"] if case["kind"] == "weights" else 0
    table, pages = _table(rng, case, room)
    T = table.shape[1] * P
    # earlier evictions leave a head's kept positions in any order behind the fixed ones
    fixed = np.minimum(case["fixed"], lens).astype(np.int32)
    seen = lens + rng.integers(0, 64, size=B).astype(np.int32)
    order = torch.rand((B, Hkv, T + 64), generator=g, device="cuda")
    ids = torch.arange(T + 64, device="cuda")
    fx = _dev(fixed)[:, None, None]
    order = torch.where(ids < fx, ids.float() - 1e6, torch.where(ids < _dev(seen)[:, None, None], order, 2.0))
    position = order.argsort(dim=-1)[..., :T].to(torch.int32).contiguous()
    # a few keys get most of the attention
    weight = torch.rand((B, Hkv, T), generator=g, device="cuda").pow_(8).mul_(50.0)
    s.update(k_cache=bf(pages, P, Hkv, D), page_table=_dev(table), kv_len=_dev(lens), seen=_dev(seen),
             max_kv_len=int(lens.max()), fixed_len=_dev(fixed), weight=weight, position=position, weight_out=torch.zeros_like(weight))
    if case["kind"] == "weights":
        N, Hq = case["N"], case["Hq"]
        alen = rng.integers(1, case["amax"] + 1, size=B).astype(np.int32)
        idx = np.full((B, N), -1, dtype=np.int32)
        for b in range(B):               # a root path: ascending node ids from a root
            idx[b, :alen[b]] = np.sort(rng.choice(N, alen[b], replace=False))
        lse = torch.randn((B, N, Hq), generator=g, device="cuda").mul_(0.05)
        lse += torch.log(_dev(lens).float() + 1.0)[:, None, None] + 0.5
        s.update(q=bf(B, N, Hq, D), lse=lse, accept_idx=_dev(idx), accept_len=_dev(alen))
    else:
        s.update(v_cache=bf(pages, P, Hkv, D), position_out=torch.zeros_like(position),
                 kept_len=torch.zeros(B, dtype=torch.int32, device="cuda"), workspace=None)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _rows(cache, table, n):
    """[B, Hkv, n, D] fp32: the first n positions' rows through the page table."""
    P = cache.shape[1]
    t = torch.arange(n, device="cuda")
    return cache[table[:, t // P].long(), t % P].permute(0, 2, 1, 3).float()


def _plain_shared(s):
    c = s["case"]
    B, N, Hq, Hkv, D = (c[k] for k in ("B", "N", "Hq", "Hkv", "D"))
    G, L = Hq // Hkv, s["max_kv_len"]
    q = s["q"].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    # ancestors: the closure of (itself, its parent) by squaring
    ids = torch.arange(N, device="cuda")
    seen = ((ids[:, None] == ids) | (s["parent"].long()[:, :, None] == ids)).float()
    for _ in range(8):
        seen = torch.matmul(seen, seen).clamp(max=1.0)
    k = torch.cat([_rows(s["k_cache"], s["page_table"], L), s["k_tree"].permute(0, 2, 1, 3).float()], 2)
    v = torch.cat([_rows(s["v_cache"], s["page_table"], L), s["v_tree"].permute(0, 2, 1, 3).float()], 2)
    x = torch.matmul(q, k.transpose(2, 3)).div_(math.sqrt(D))
    prefix = (torch.arange(L, device="cuda") < s["kv_len"][:, None])[:, None, :].expand(B, N * G, L)
    visible = torch.cat([prefix, (seen > 0).repeat_interleave(G, dim=1)], 2)[:, None]
    x = x.masked_fill_(~visible, -math.inf)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    out = (torch.matmul(x, v) / total).view(B, Hkv, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)
    lse = (m + total.log()).view(B, Hkv, N, G).permute(0, 2, 1, 3).reshape(B, N, Hq)
    if s["num_nodes"] is not None:
        pad = ids >= s["num_nodes"][:, None]
        out = out.masked_fill(pad[:, :, None, None], 0.0)
        lse = lse.masked_fill(pad[:, :, None], -math.inf)
    return out.to(BF16), lse


def _plain_weights(s):
    c = s["case"]
    B, Hq, Hkv, D, T = c["B"], c["Hq"], c["Hkv"], c["D"], s["weight"].shape[2]
    G, A = Hq // Hkv, int(s["accept_len"].max())
    at = torch.arange(A, device="cuda")
    idx = s["accept_idx"][:, :A].clamp(min=0).long()
    b = torch.arange(B, device="cuda")[:, None]
    q = s["q"][b, idx].float().view(B, A, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, A * G, D)
    lse = s["lse"][b, idx].view(B, A, Hkv, G).permute(0, 2, 1, 3).reshape(B, Hkv, A * G, 1)
    x = torch.matmul(q, _rows(s["k_cache"], s["page_table"], T).transpose(2, 3)).div_(math.sqrt(D))
    x = x.sub_(lse).exp_()
    # row j sees the prefix and the path up to itself
    t, L = torch.arange(T, device="cuda"), s["kv_len"][:, None, None]
    live = (t <= L + at[:, None]) & (at[:, None] < s["accept_len"][:, None, None])
    mass = x.masked_fill_(~live.repeat_interleave(G, dim=1)[:, None], 0.0).sum(2)
    end = L + s["accept_len"][:, None, None]
    w = torch.where(t < L, s["weight"] + mass.masked_fill(t < s["fixed_len"][:, None, None], 0.0), mass)
    new = (t >= L) & (t < end)
    weight = torch.where(t < end, w, s["weight_out"])
    position = torch.where(new, (s["seen"][:, None, None] + t - L).to(torch.int32), s["position"])
    return weight, position


def _plain_evict(s):
    c = s["case"]
    T, P = s["weight"].shape[2], c["P"]
    t = torch.arange(T, device="cuda")
    L, fixed = s["kv_len"][:, None, None], s["fixed_len"][:, None, None]
    keep = torch.minimum(L, fixed.clamp(min=c["budget"]))
    kind = (s["position"] >= s["seen"][:, None, None] - c["recent"]).int()
    kind = torch.where(t < fixed, 2, torch.where(t < L, kind, -1))
    order = s["weight"].argsort(dim=-1, descending=True, stable=True)
    order = order.gather(-1, kind.gather(-1, order).argsort(dim=-1, descending=True, stable=True))
    rank = torch.empty_like(order).scatter_(-1, order, t.expand_as(order))
    kept = rank < keep
    hole, src = ~kept & (t < keep), kept & (t >= keep)
    # the k-th hole takes the k-th kept slot past the kept length: both lists in slot order
    hb, hg, ht = hole.nonzero(as_tuple=True)
    _, _, st = src.nonzero(as_tuple=True)
    weight = torch.where(t < keep, s["weight"], s["weight_out"])
    position = torch.where(t < keep, s["position"], s["position_out"])
    weight[hb, hg, ht] = s["weight"][hb, hg, st]
    position[hb, hg, ht] = s["position"][hb, hg, st]
    table = s["page_table"].long()
    for cache in (s["k_cache"], s["v_cache"]):
        cache[table[hb, ht // P], ht % P, hg] = cache[table[hb, st // P], st % P, hg]
    return s["k_cache"], s["v_cache"], weight, position, keep.view(-1).to(torch.int32)


def run(state):
    s, c = state, state["case"]
    if c["kind"] == "shared":
        if own:
            import paper_2602_21224_amd as T
            if s["workspace"] is None:
                s["workspace"] = torch.empty(T.shared_attention_workspace_size(
                    c["B"], c["N"], c["Hq"], c["Hkv"], c["D"], c["groups"]), dtype=torch.uint8, device="cuda")
            return T.tree_verify_attention_shared(
                s["q"], s["k_tree"], s["v_tree"], s["k_cache"], s["v_cache"], s["page_table"], s["kv_len"],
                s["parent"], s["group_start"], s["shared_len"], max_kv_len=s["max_kv_len"],
                num_nodes=s["num_nodes"], out=s["out"], lse=s["lse"], workspace=s["workspace"])
        return _plain_shared(s)
    if c["kind"] == "weights":
        if own:
            import paper_2602_21224_amd as T
            return T.kv_accumulate_weights(
                s["q"], s["lse"], s["k_cache"], s["page_table"], s["kv_len"], s["accept_idx"], s["accept_len"],
                s["weight"], s["position"], s["seen"], max_kv_len=s["max_kv_len"], fixed_len=s["fixed_len"],
                weight_out=s["weight_out"])
        return _plain_weights(s)
    if own:
        import paper_2602_21224_amd as T
        if s["workspace"] is None:
            s["workspace"] = torch.empty(T.evict_workspace_size(c["B"], c["Hkv"], s["page_table"].shape[1], c["P"]),
                                         dtype=torch.uint8, device="cuda")
        weight, position, kept = T.kv_evict(
            s["weight"], s["position"], s["k_cache"], s["v_cache"], s["page_table"], s["kv_len"], s["seen"],
            max_kv_len=s["max_kv_len"], budget=c["budget"], recent=c["recent"], fixed_len=s["fixed_len"],
            weight_out=s["weight_out"], position_out=s["position_out"], kept_len=s["kept_len"],
            workspace=s["workspace"])
        return s["k_cache"], s["v_cache"], weight, position, kept
    return _plain_evict(s)


# ---------------------------------------------------------------------------
# the definitions in 64 bits, one sequence at a time
# ---------------------------------------------------------------------------

def _exact_attention(s):
    c = s["case"]
    N, Hq, Hkv, D, P = (c[k] for k in ("N", "Hq", "Hkv", "D", "P"))
    G = Hq // Hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    parent, lens = s["parent"].cpu().numpy(), s["kv_len"].tolist()
    for b, L in enumerate(lens):
        n = N if s["num_nodes"] is None else int(s["num_nodes"][b])
        sees = np.zeros((n, n), dtype=bool)
        for i in range(n):               # a node's root path is its parent's and itself
            if parent[b, i] >= 0:
                sees[i] = sees[parent[b, i]]
            sees[i, i] = True
        sees = _dev(sees)
        pages = s["page_table"][b, :-(-L // P)].long()
        kp = s["k_cache"][pages].reshape(-1, Hkv, D)[:L].double()
        vp = s["v_cache"][pages].reshape(-1, Hkv, D)[:L].double()
        for h in range(Hkv):
            for j in range(h * G, h * G + G):
                q = s["q"][b, :n, j].double()
                xp = (q @ kp[:, h].T) / math.sqrt(D)
                xt = (q @ s["k_tree"][b, :n, h].double().T) / math.sqrt(D)
                xt = torch.where(sees, xt, torch.full_like(xt, -math.inf))
                z = torch.logsumexp(torch.cat([xp, xt], 1), 1)
                out[b, :n, j] = (torch.exp(xp - z[:, None]) @ vp[:, h]
                                 + torch.exp(xt - z[:, None]) @ s["v_tree"][b, :n, h].double())
                lse[b, :n, j] = z
    return out, lse


def _exact_weights(s):
    c = s["case"]
    Hq, Hkv, D, P = (c[k] for k in ("Hq", "Hkv", "D", "P"))
    G = Hq // Hkv
    weight, position = s["weight_out"].double().clone(), s["position"].clone()
    for b, L in enumerate(s["kv_len"].tolist()):
        n, f = int(s["accept_len"][b]), int(s["fixed_len"][b])
        nodes = s["accept_idx"][b, :n].long()
        pages = s["page_table"][b, :-(-(L + n) // P)].long()
        k = s["k_cache"][pages].reshape(-1, Hkv, D)[:L + n].double()
        for h in range(Hkv):
            total = torch.zeros(L + n, dtype=torch.float64, device="cuda")
            for j in range(n):
                q = s["q"][b, nodes[j], h * G:h * G + G].double()
                z = s["lse"][b, nodes[j], h * G:h * G + G].double()
                x = (k[:L + j + 1, h] @ q.T) / math.sqrt(D)
                total[:L + j + 1] += torch.exp(x - z).sum(1)
            total[:f] = 0.0
            total[:L] += s["weight"][b, h, :L].double()
            weight[b, h, :L + n] = total
            position[b, h, L:L + n] = int(s["seen"][b]) + torch.arange(n, device="cuda", dtype=torch.int32)
    return weight, position


def _exact_evict(s):
    c = s["case"]
    k, v = s["k_cache"].clone(), s["v_cache"].clone()
    table = s["page_table"].cpu().numpy().astype(np.int64)
    win, pin = s["weight"].cpu().numpy(), s["position"].cpu().numpy()
    wout, pout = np.zeros_like(win), np.zeros_like(pin)
    kept = np.zeros(c["B"], dtype=np.int32)
    for b, L in enumerate(s["kv_len"].tolist()):
        f, seen = int(s["fixed_len"][b]), int(s["seen"][b])
        n = kept[b] = min(L, max(c["budget"], f))
        t = np.arange(L)
        for h in range(c["Hkv"]):
            w, p = win[b, h, :L], pin[b, h, :L]
            kind = np.where(t < f, 0, np.where(p >= seen - c["recent"], 1, 2))
            best = np.lexsort((t, -w.astype(np.float64), kind))[:n]
            stay = np.zeros(L, dtype=bool)
            stay[best] = True
            dst, src = np.nonzero(~stay[:n])[0], n + np.nonzero(stay[n:])[0]
            wout[b, h, :n], pout[b, h, :n] = w[:n], p[:n]
            wout[b, h, dst], pout[b, h, dst] = w[src], p[src]
            to, at = (_dev(np.stack([table[b, x // c["P"]], x % c["P"]])) for x in (dst, src))
            for cache in (k, v):
                cache[to[0], to[1], h] = cache[at[0], at[1], h]
    return k.double(), v.double(), _dev(wout).double(), _dev(pout), _dev(kept)


def exact(case, seed):
    s = prepare(case, seed)
    return {"shared": _exact_attention, "weights": _exact_weights, "evict": _exact_evict}[case["kind"]](s)


def work(case):
    """Each input read once and each output written once, at the mean lengths."""
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    L = (case["lo"] + case["hi"]) / 2
    if case["kind"] == "shared":
        N, Hq, S = case["N"], case["Hq"], (case["slo"] + case["shi"]) / 2
        n = N * (2 / 3 if case["ragged"] else 1)
        keys = S * case["groups"] + (L + n) * B
        return {"bytes": keys * Hkv * D * 4 + B * N * Hq * (D * 4 + 4), "flops": 4.0 * B * n * Hq * D * (S + L + n)}
    live = L - min(case["fixed"], L)
    if case["kind"] == "weights":
        a = (1 + case["amax"]) / 2
        return {"bytes": B * Hkv * ((live + a) * D * 2 + (L + a) * 8) + B * a * case["Hq"] * (D * 2 + 4),
                "flops": 2.0 * B * a * case["Hq"] * (live + a) * D}
    over = max(0.0, L - max(case["budget"], case["fixed"]))
    if case["lo"] < case["budget"] < case["hi"]:
        over = (case["hi"] - case["budget"]) ** 2 / 2 / (case["hi"] - case["lo"])
    moved = over * (L - over) / L
    return {"bytes": B * Hkv * (L * 8 + (L - over) * 8 + moved * D * 8), "flops": B * Hkv * L}
