"""Cases of the operators for long contexts: a K/V cache held in 4 bits, the rows
written into it, tree attention over it, and tree attention inside a sliding window
with a few first tokens that stay visible.

A serving loop that keeps its K/V cache in blocks of 32 four-bit values with a shared
power of two puts prompts, single tokens and accepted paths into it with `kv4_write`
and verifies its draft trees over it with `tree_verify_attention_kv4`; a model whose
layers look back over a window only calls `tree_verify_attention_window` on its bf16
cache (or gives the same window to the call on 4 bits), with the pages behind the
window given back. The listed cases take each call at the sizes of this repository's
presets and between them; the drawn ones spread over the same ranges. Workspaces and
output buffers are kept between calls, as a serving loop keeps them.
"""
import math

import numpy as np
import torch

own = False

BF16 = torch.bfloat16


def listed():
    return [
        # One token of one sequence enters the cache.
        dict(name="write_one", kind="write", B=1, T=1, Hkv=8, D=64, P=16, lo=128, hi=128, path=False, ragged=False),
        # The accepted paths of a verified batch, up to 8 of 64 nodes each.
        dict(name="write_path_b16", kind="write", B=16, T=64, Hkv=8, D=128, P=16, lo=1024, hi=4096, path=True,
             ragged=True),
        # Ragged prompts, five KV heads, one-token pages.
        dict(name="write_ragged_d64", kind="write", B=5, T=777, Hkv=5, D=64, P=1, lo=0, hi=301, path=False, ragged=True),
        # Long prompts, whole.
        dict(name="write_prompts_b4", kind="write", B=4, T=8192, Hkv=8, D=128, P=16, lo=0, hi=0, path=False,
             ragged=False),
        # Plain decoding of one request: what a single user waits for.
        dict(name="kv4_decode_b1", kind="kv4", B=1, N=1, Hq=32, Hkv=8, D=128, P=16, lo=2048, hi=2048, window=0, sinks=0,
             tree="chain", ragged=False),
        # Plain decoding of a full batch.
        dict(name="kv4_decode_b64", kind="kv4", B=64, N=1, Hq=32, Hkv=8, D=128, P=16, lo=2048, hi=8192, window=0,
             sinks=0, tree="chain", ragged=False),
        # Multi-head attention with the narrow 12-token trees that the method verifies.
        dict(name="kv4_mha_b16", kind="kv4", B=16, N=12, Hq=32, Hkv=32, D=128, P=16, lo=256, hi=2048, window=0, sinks=0,
             tree="capped", ragged=False),
        # Grouped-query attention of an 8B-shaped layer, 64-node trees.
        dict(name="kv4_gqa_b16", kind="kv4", B=16, N=64, Hq=32, Hkv=8, D=128, P=16, lo=1024, hi=4096, window=0, sinks=0,
             tree="capped", ragged=False),
        # Few requests with very long contexts, a short chain of draft tokens each.
        dict(name="kv4_long_b4", kind="kv4", B=4, N=4, Hq=32, Hkv=8, D=128, P=64, lo=98304, hi=131072, window=0, sinks=0,
             tree="chain", ragged=False),
        # Small: forests of different sizes over 4 bits inside a window, head size 64,
        # one-token pages, three heads per KV head, odd lengths.
        dict(name="kv4_window_d64", kind="kv4", B=5, N=45, Hq=24, Hkv=8, D=64, P=1, lo=300, hi=777, window=201, sinks=5,
             tree="forest", ragged=True),
        # Plain decoding inside a window, long contexts.
        dict(name="window_decode_b32", kind="window", B=32, N=1, Hq=32, Hkv=8, D=128, P=16, lo=4096, hi=32768, window=4096,
             sinks=4, tree="chain", ragged=False),
        # 64-node trees inside a window.
        dict(name="window_gqa_b16", kind="window", B=16, N=64, Hq=32, Hkv=8, D=128, P=16, lo=1024, hi=32768, window=2048,
             sinks=16, tree="capped", ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "kv4", "kv4", "kv4", "window", "window"])
    while True:
        Hkv = rng.choice([2, 4, 5, 8, 8, 16, 32])
        D, P = rng.choice([64, 128, 128]), rng.choice([1, 2, 8, 16, 16, 16, 32, 64, 256])
        B = _log_int(rng, 1, 96)
        if kind == "write":
            path = rng.random() < 0.4
            hi = rng.choice([0, _log_int(rng, 1, 4096)])
            c = dict(kind=kind, B=B, T=_log_int(rng, 1, 256 if path else 8192), Hkv=Hkv, D=D, P=P,
                     lo=rng.choice([hi, hi // 2]), hi=hi, path=path, ragged=path or rng.random() < 0.5)
            if B * (c["T"] + hi) * Hkv * D > 3e7:
                continue
        else:
            N, hi = rng.choice([1, 1, _log_int(rng, 2, 256)]), _log_int(rng, 64, 131072)
            window = rng.choice([0, _log_int(rng, 16, 8192)]) if kind == "kv4" else _log_int(rng, 16, 8192)
            c = dict(kind=kind, B=B, N=N, Hq=Hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), Hkv=Hkv, D=D, P=P,
                     lo=rng.choice([hi, hi // 2, hi // 8]), hi=hi, window=window,
                     sinks=rng.choice([0, 1, 4, 16, 100]) if window else 0,
                     tree=rng.choice(["forest", "capped", "chain"]), ragged=N >= 12 and rng.random() < 0.3)
            if N * c["Hq"] > 2048 * Hkv or work(c)["flops"] > 5e10 or B * hi * Hkv * D > 5e8:
                continue
            if B * c["Hq"] * N * hi > 1.2e9 or work(c)["bytes"] > 3e8:
                continue
        return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

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


def _table(rng, lens, room, P, window=0, sinks=0):
    """Page table [B, max_pages] of random pages with `room` more tokens behind each
    sequence, and the number of pages. Pages wholly behind a sequence's window, and not
    of its first `sinks` tokens, have been given back (-1)."""
    need = -(-(lens.astype(np.int64) + room) // P)
    per = max(1, int(need.max()))
    page = np.arange(per)[None, :]
    held = page < need[:, None]
    if window:
        first = np.maximum(lens.astype(np.int64) + 1 - window, 0)
        held &= (page < -(-sinks // P)) | (page >= (first // P)[:, None])
    table = np.full((len(lens), per), -1, dtype=np.int32)
    n = int(held.sum())
    table[held] = rng.permutation(n).astype(np.int32)
    return table, max(n, 1)


def _cache4(g, pages, Hkv, P, D):
    """Codes of K and of V and their scales, of normal rows; some channels of K are larger."""
    codes = []
    scales = torch.empty((pages, Hkv, P, 2, D // 32), dtype=torch.uint8, device="cuda")
    gain = torch.randn(D, generator=g, device="cuda").mul_(0.4).exp_()
    step = max(1, 2 ** 25 // (Hkv * P * D))
    for i in range(2):
        c = torch.empty((pages, Hkv, P, D // 2), dtype=torch.uint8, device="cuda")
        for a in range(0, pages, step):
            x = torch.randn((min(step, pages - a), Hkv, P, D), generator=g, device="cuda")
            c[a:a + step], scales[a:a + step, :, :, i] = _to4((x * gain if i == 0 else x).to(BF16))
        codes.append(c)
    return codes[0], codes[1], scales


def prepare(case, seed):
    B, Hkv, D, P = (case[k] for k in ("B", "Hkv", "D", "P"))
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda")
    g.manual_seed(seed)
    bf = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=BF16)  # noqa: E731
    lens = rng.integers(case["lo"], case["hi"] + 1, size=B).astype(np.int32)
    s = dict(case=case)
    if case["kind"] == "write":
        T = case["T"]
        table, _ = _table(rng, lens, T, P)
        pages = B * -(-(case["hi"] + T) // P)          # a pool of one size, whatever the lengths
        counts = np.full(B, T, dtype=np.int32)
        idx = None
        if case["path"]:                 # a root path: ascending node ids
            counts = rng.integers(1, min(T, 8) + 1, size=B).astype(np.int32)
            idx = np.full((B, T), -1, dtype=np.int32)
            for b in range(B):
                idx[b, :counts[b]] = np.sort(rng.choice(T, counts[b], replace=False))
        elif case["ragged"]:
            counts = rng.integers(T // 2, T + 1, size=B).astype(np.int32)
        zeros = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device="cuda")  # noqa: E731
        s.update(k=bf(B, T, Hkv, D), v=bf(B, T, Hkv, D), k4=zeros(pages, Hkv, P, D // 2), v4=zeros(pages, Hkv, P, D // 2),
                 scales=zeros(pages, Hkv, P, 2, D // 32), page_table=_dev(table), start=_dev(lens),
                 idx=None if idx is None else _dev(idx), count=_dev(counts) if case["ragged"] else None,
                 k_held=torch.zeros((B, T, Hkv, D), dtype=BF16, device="cuda"),
                 v_held=torch.zeros((B, T, Hkv, D), dtype=BF16, device="cuda"))
        return s
    N, Hq = case["N"], case["Hq"]
    table, pages = _table(rng, lens, N, P, case["window"], case["sinks"])
    parent, counts = _parents(rng, case)
    s.update(q=bf(B, N, Hq, D), k_tree=bf(B, N, Hkv, D), v_tree=bf(B, N, Hkv, D), page_table=_dev(table),
             kv_len=_dev(lens), parent=_dev(parent), num_nodes=_dev(counts) if case["ragged"] else None,
             max_kv_len=int(lens.max()), out=torch.empty((B, N, Hq, D), dtype=BF16, device="cuda"),
             lse=torch.empty((B, N, Hq), dtype=torch.float32, device="cuda"), workspace=None)
    if case["kind"] == "kv4":
        s["k4"], s["v4"], s["scales"] = _cache4(g, pages, Hkv, P, D)
    else:
        s["k_cache"], s["v_cache"] = bf(pages, P, Hkv, D), bf(pages, P, Hkv, D)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _to4(x):
    """Codes [..., D / 2] and scale bytes [..., D / 32] of rows x [..., D]: per block of 32
    the smallest power of two 2^e (e >= -126) with which the largest magnitude is at most
    7, then each value to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code)."""
    x = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1))               # m in [1/2, 1)
    e = torch.clamp(e - 3 + (m > 0.875).int(), min=-126)
    y = torch.ldexp(x.abs(), -e[..., None])
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    code = (code + 8 * torch.signbit(x)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _from4(codes, scales):
    """fp32 rows [..., D] that codes [..., D / 2] and scale bytes [..., D / 32] stand for."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    byte = torch.arange(256, device="cuda")
    both = torch.stack([grid[byte % 16], grid[byte // 16]], 1)
    x = both[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    return (x * torch.exp2(scales.float() - 127)[..., None]).flatten(-2)


def _plain_write(s):
    T, P = s["case"]["T"], s["case"]["P"]
    j = torch.arange(T, device="cuda")
    live = (j < s["count"][:, None]) if s["count"] is not None else (j >= 0).expand(s["case"]["B"], T)
    b, j = live.nonzero(as_tuple=True)
    src = j if s["idx"] is None else s["idx"][b, j].long()
    pos = s["start"][b] + j
    page, slot = s["page_table"][b, pos // P].long(), pos % P
    for i, (x, codes, held) in enumerate(((s["k"], s["k4"], s["k_held"]), (s["v"], s["v4"], s["v_held"]))):
        c, e = _to4(x[b, src])
        codes[page, :, slot] = c
        s["scales"][page, :, slot, i] = e
        held[b, j] = _from4(c, e).to(BF16)
    return s["k_held"], s["v_held"], s["k4"], s["v4"], s["scales"]


def _plain_attention(s):
    c = s["case"]
    B, N, Hq, Hkv, D, P = (c[k] for k in ("B", "N", "Hq", "Hkv", "D", "P"))
    G, L = Hq // Hkv, s["max_kv_len"]
    t = torch.arange(L, device="cuda")
    page = s["page_table"][:, t // P].long().clamp(min=0)
    if c["kind"] == "kv4":
        both = s["scales"][page, :, t % P]
        kp, vp = _from4(s["k4"][page, :, t % P], both[..., 0, :]), _from4(s["v4"][page, :, t % P], both[..., 1, :])
    else:
        kp, vp = s["k_cache"][page, t % P].float(), s["v_cache"][page, t % P].float()
    k = torch.cat([kp, s["k_tree"].float()], 1).permute(0, 2, 1, 3)
    v = torch.cat([vp, s["v_tree"].float()], 1).permute(0, 2, 1, 3)
    q = s["q"].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    # ancestors: the closure of (itself, its parent) by squaring
    ids = torch.arange(N, device="cuda")
    seen = ((ids[:, None] == ids) | (s["parent"].long()[:, :, None] == ids)).float()
    for _ in range(8):
        seen = torch.matmul(seen, seen).clamp(max=1.0)
    seen = seen > 0
    # positions: the prefix's, then the nodes', each at its depth behind the prefix
    at = s["kv_len"][:, None] + seen.sum(-1) - 1
    key = torch.cat([t.expand(B, L), at], 1)[:, None]
    visible = torch.cat([(t < s["kv_len"][:, None])[:, None].expand(B, N, L), seen], 2)
    if c["window"]:
        visible = visible & ((key < c["sinks"]) | (key > at[:, :, None] - c["window"]))
    x = torch.matmul(q, k.transpose(2, 3)).div_(math.sqrt(D))
    x = x.masked_fill_(~visible.repeat_interleave(G, dim=1)[:, None], -math.inf)
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


def run(state):
    s, c = state, state["case"]
    if c["kind"] == "write":
        if own:
            import paper_2602_21224_amd as T
            T.kv4_write(s["k"], s["v"], s["k4"], s["v4"], s["scales"], s["page_table"], s["start"], idx=s["idx"],
                        count=s["count"], k_held=s["k_held"], v_held=s["v_held"])
            return s["k_held"], s["v_held"], s["k4"], s["v4"], s["scales"]
        return _plain_write(s)
    if own:
        import paper_2602_21224_amd as T
        if s["workspace"] is None:
            size = T.kv4_attention_workspace_size if c["kind"] == "kv4" else T.window_attention_workspace_size
            s["workspace"] = torch.empty(size(c["B"], c["N"], c["Hq"], c["Hkv"], c["D"]), dtype=torch.uint8, device="cuda")
        more = dict(max_kv_len=s["max_kv_len"], window=c["window"], sinks=c["sinks"], num_nodes=s["num_nodes"], out=s["out"],
                    lse=s["lse"], workspace=s["workspace"])
        if c["kind"] == "kv4":
            return T.tree_verify_attention_kv4(s["q"], s["k_tree"], s["v_tree"], s["k4"], s["v4"], s["scales"],
                                               s["page_table"], s["kv_len"], s["parent"], **more)
        return T.tree_verify_attention_window(s["q"], s["k_tree"], s["v_tree"], s["k_cache"], s["v_cache"], s["page_table"],
                                              s["kv_len"], s["parent"], **more)
    return _plain_attention(s)


# ---------------------------------------------------------------------------
# the definitions in 64 bits, one sequence at a time
# ---------------------------------------------------------------------------

def _held(x):
    """The values that rows x [n, Hkv, D] are held as: each block of 32 on the grid of its
    power of two, by distance, the even one of two equally near."""
    a = np.abs(x).reshape(-1, 32)
    e = np.full(len(a), -126)
    top = a.max(1)
    while (top > 7 * 2.0 ** e).any():
        e += top > 7 * 2.0 ** e
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    y = a / 2.0 ** e[:, None]
    low = np.clip(np.searchsorted(grid, y, side="right") - 1, 0, 6)
    up = grid[low + 1] - y
    down = y - grid[low]
    take = low + ((up < down) | ((up == down) & (low % 2 == 1)))
    return (np.sign(x).reshape(-1, 32) * grid[take] * 2.0 ** e[:, None]).reshape(x.shape)


def _exact_write(s):
    outs = []
    count = s["case"]["T"] if s["count"] is None else s["count"].cpu().numpy()
    for x in (s["k"], s["v"]):
        x = x.double().cpu().numpy()
        held = np.zeros(x.shape)
        for b in range(len(x)):
            n = int(np.broadcast_to(count, len(x))[b])
            rows = np.arange(n) if s["idx"] is None else s["idx"][b, :n].cpu().numpy()
            held[b, :n] = _held(x[b, rows])
        outs.append(_dev(held))
    return outs[0], outs[1], None, None, None


def _values(codes, exps):
    """fp64 rows of codes [n, D / 2] and scale bytes [n, D / 32]: sign, two bits of exponent
    and one of mantissa each, exponent 0 without the leading one."""
    n = torch.stack([codes.long() & 15, codes.long() >> 4], -1).flatten(1)
    e, m = (n >> 1) & 3, (n & 1).double()
    x = torch.where(e == 0, m / 2, (1 + m / 2) * torch.pow(2.0, (e - 1).double())) * (1 - 2 * (n >> 3)).double()
    return x * torch.pow(2.0, exps.double() - 127).repeat_interleave(32, dim=1)


def _exact_attention(s):
    c = s["case"]
    N, Hq, Hkv, D, P, W, S = (c[k] for k in ("N", "Hq", "Hkv", "D", "P", "window", "sinks"))
    G = Hq // Hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    parent, table = s["parent"].cpu().numpy(), s["page_table"].cpu().numpy()
    for b, L in enumerate(s["kv_len"].tolist()):
        n = N if s["num_nodes"] is None else int(s["num_nodes"][b])
        first = max(0, L + 1 - W) if W else 0                       # of the keys that a root sees
        pos = np.concatenate([np.arange(min(S if W else 0, first)), np.arange(first, L)]).astype(np.int64)
        depth, sees = np.zeros(n, dtype=np.int64), np.zeros((n, len(pos) + n), dtype=bool)
        for i in range(n):
            depth[i] = 0 if parent[b, i] < 0 else depth[parent[b, i]] + 1
            a = i
            while a >= 0:                                           # its root path
                sees[i, len(pos) + a] = not W or depth[i] - depth[a] < W or L + depth[a] < S
                a = parent[b, a]
            sees[i, :len(pos)] = True if not W else (pos < S) | (L + depth[i] - pos < W)
        sees = _dev(sees)
        page, slot = _dev(table[b, pos // P].astype(np.int64)), _dev(pos % P)
        for h in range(Hkv):
            if c["kind"] == "kv4":
                kp, vp = (_values(s[name][page, h, slot], s["scales"][page, h, slot, i])
                          for i, name in enumerate(("k4", "v4")))
            else:
                kp, vp = s["k_cache"][page, slot, h].double(), s["v_cache"][page, slot, h].double()
            k = torch.cat([kp.view(-1, D), s["k_tree"][b, :n, h].double()])
            v = torch.cat([vp.view(-1, D), s["v_tree"][b, :n, h].double()])
            for j in range(h * G, h * G + G):
                x = (s["q"][b, :n, j].double() @ k.T) / math.sqrt(D)
                x = torch.where(sees, x, torch.full_like(x, -math.inf))
                z = torch.logsumexp(x, 1)
                out[b, :n, j], lse[b, :n, j] = torch.exp(x - z[:, None]) @ v, z
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_write(s) if case["kind"] == "write" else _exact_attention(s)


def work(case):
    """Each input read once and each output written once, at the mean lengths."""
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    row4 = 2 * (D // 2 + D // 32)                      # K and V of one key and KV head
    if case["kind"] == "write":
        T = case["T"]
        n = (1 + min(T, 8)) / 2 if case["path"] else 0.75 * T if case["ragged"] else T
        return {"bytes": B * n * Hkv * (8 * D + row4), "flops": B * n * Hkv * D * 4}
    N, Hq, W, S = (case[k] for k in ("N", "Hq", "window", "sinks"))
    n = N * (2 / 3 if case["ragged"] else 1)
    seen = lambda L: L if not W else min(L, W - 1 + S)  # noqa: E731
    keys = sum(seen(case["lo"] + (case["hi"] - case["lo"]) * (i + 0.5) / 64) for i in range(64)) / 64
    row = row4 if case["kind"] == "kv4" else 4 * D
    return {"bytes": B * Hkv * (keys * row + n * 4 * D) + B * N * Hq * (D * 4 + 4), "flops": 4.0 * B * n * Hq * D * (keys + n)}
