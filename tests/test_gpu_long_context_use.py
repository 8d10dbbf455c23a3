"""The long-context operators as programs use them: large pools, other streams with work
pending, graphs that share a workspace, large batches, padded ones."""
import numpy as np
import pytest
import torch

from oracle import long_context as O
from paper_2602_21224_amd import workloads as W
from tests import gpu_util as U
from tests import long_util as LU
from tests.test_gpu_cache_streams import LONG, pending
from tests.test_gpu_cache_streams import same as same_all

pytestmark = pytest.mark.gpu


def call(T, which, d, cache, hint, **kw):
    """One of the two attentions over tensors that are on the device."""
    f = T.tree_verify_attention_window if which == "window" else T.tree_verify_attention_kv4
    return f(d["q"], d["k_tree"], d["v_tree"], *cache, d["page_table"], d["kv_len"], d["parent"], max_kv_len=hint,
             num_nodes=d["num_nodes"], **kw)


def setup(which, seed=70, window=90, sinks=3, **kw):
    args = dict(B=3, N=14, Hq=8, Hkv=2, D=128, P=16, lens=[900, 0, 333])
    args.update(kw)
    w = LU.workload(seed, **args, window=window, sinks=sinks)
    d = U.upload(w)
    bits = None if which == "window" else LU.cache4(w)
    cache = [d["k_cache"], d["v_cache"]] if bits is None else [U.dev(a) for a in bits]
    return w, d, cache, bits, dict(window=window, sinks=sinks)


def far_pool(small, pages):
    """A pool of `pages` pages whose last ones are `small`'s; the others are never touched."""
    big = torch.empty((pages, *small.shape[1:]), dtype=small.dtype, device="cuda")
    big[pages - len(small):].copy_(small)
    return big


def far_pages(table, pool, pages):
    """The same table for pages at the end of the larger pool (bad ids stay bad)."""
    t = table.astype(np.int64)
    return np.where((t >= 0) & (t < pool), t + pages - pool, t).clip(-1, 0x7FFFFFFF).astype(np.int32)


@pytest.mark.parametrize("N,P", [(2, 256), (3, 4), (40, 256), (60, 2)])
def test_pages_past_4_gib(N, P):
    """Codes and scale bytes past 2^32 bytes from the pool's start (72 GB of pools, of which a
    few pages are used), each kernel, and the write there."""
    T = U.require_gpu()
    Hkv, D = 2, 128
    pages = (1 << 29) // (Hkv * P) + 4096        # 2^29 rows of 64 bytes of codes and 8 of scales
    print(f"N={N} P={P}: {pages} pages", flush=True)
    w, d, _, bits, kw = setup("4 bits", 71 + N, 0, 0, B=2, N=N, Hkv=Hkv, Hq=8, D=D, P=P, lens=[700, 65])
    small = [U.dev(a) for a in bits]
    d["page_table"] = U.dev(far_pages(w.page_table, len(w.k_cache), pages))
    pool = [far_pool(a, pages) for a in small]
    out, lse = call(T, "4 bits", d, pool, w.max_kv_len, **kw)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, 0, 0, bits), "far")
    start = U.dev(np.array([3, 0], np.int32))    # over the prefixes' first rows
    near = U.dev(w.page_table)
    T.kv4_write(d["k_tree"], d["v_tree"], *small, near, start)
    T.kv4_write(d["k_tree"], d["v_tree"], *pool, d["page_table"], start)
    for a, b in zip(pool, small):
        assert torch.equal(a[pages - len(b):], b)


@pytest.mark.parametrize("N", [1, 40])
def test_window_over_pages_past_4_gib(N):
    T = U.require_gpu()
    pages = (1 << 32) // (16 * 2 * 64 * 2) + 4096
    w, d, cache, _, kw = setup("window", 75, 100, 4, B=2, N=N, Hkv=2, Hq=8, D=64, P=16, lens=[700, 65])
    d["page_table"] = U.dev(far_pages(w.page_table, len(w.k_cache), pages))
    out, lse = call(T, "window", d, [far_pool(a, pages) for a in cache], w.max_kv_len, **kw)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, 100, 4), "far")


@pytest.mark.parametrize("N", [14, 60])
@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_own_tensors_are_not_the_current_streams(which, N):
    T = U.require_gpu()
    w, d, cache, _, kw = setup(which, N=N)
    want = [t.clone() for t in call(T, which, d, cache, w.max_kv_len, **kw)]
    size = (T.window_attention_workspace_size if which == "window" else T.kv4_attention_workspace_size)(3, N, 8, 2, 128)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    pending(want[0].nbytes, want[1].nbytes, size)
    got = call(T, which, d, cache, w.max_kv_len, **kw, stream=side)
    torch.cuda.synchronize()
    assert same_all(got, want)


@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_results_last_until_the_current_stream_is_done_with_them(which):
    T = U.require_gpu()
    w, d, cache, _, kw = setup(which)
    other = dict(d, q=d["q"] * 2)
    want = call(T, which, d, cache, w.max_kv_len, **kw)[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, lse = call(T, which, d, cache, w.max_kv_len, **kw, stream=side)
    side.synchronize()
    torch.cuda._sleep(LONG)
    late = out.clone()                   # still to come when `out` is freed
    del out, lse
    call(T, which, other, cache, w.max_kv_len, **kw, stream=side)
    torch.cuda.synchronize()
    assert same_all([late], [want])


@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_two_streams_at_once(which):
    T = U.require_gpu()
    runs = [setup(which, 76 + i, N=n) for i, n in enumerate((5, 60))]
    want = [call(T, which, d, c, w.max_kv_len, **kw) for w, d, c, _, kw in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        for s, (w, d, c, _, kw) in zip(streams, runs):
            got.append(call(T, which, d, c, w.max_kv_len, **kw, stream=s))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert same_all(g, want[i % 2]), i


@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_two_graphs_share_a_workspace(which):
    """Replayed in turn on one stream, with the workspace overwritten between."""
    T = U.require_gpu()
    runs = [setup(which, 78 + i, N=n) for i, n in enumerate((5, 60))]
    size = T.window_attention_workspace_size if which == "window" else T.kv4_attention_workspace_size
    ws = torch.empty(max(size(w.B, w.N, w.Hq, w.Hkv, w.D) for w, *_ in runs), dtype=torch.uint8, device="cuda")
    want = [[t.clone() for t in call(T, which, d, c, w.max_kv_len, **kw)] for w, d, c, _, kw in runs]
    outs = [[torch.empty_like(t) for t in x] for x in want]
    torch.cuda.synchronize()
    graphs, stream = [], torch.cuda.Stream()
    for (w, d, c, _, kw), o in zip(runs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(stream), torch.cuda.graph(g, stream=stream):
            call(T, which, d, c, w.max_kv_len, **kw, out=o[0], lse=o[1], workspace=ws)
        graphs.append(g)
    for k in range(5):
        for i in (0, 1) if k % 2 else (1, 0):
            for t in outs[i]:
                t.fill_(3.0)
            ws.fill_(0xFF)
            graphs[i].replay()
        torch.cuda.synchronize()
        assert same_all(outs[0], want[0]) and same_all(outs[1], want[1]), k


@pytest.mark.parametrize("which", ["window", "4 bits"])
@pytest.mark.parametrize("B,N,lens", [(1024, 1, (0, 40)), (300, 7, (0, 200)), (130, 33, (0, 90))])
def test_large_batches(which, B, N, lens):
    """Many short sequences, some of them empty and without nodes."""
    T = U.require_gpu()
    w, d, cache, bits, kw = setup(which, 81, 30, 2, B=B, N=N, Hq=4, Hkv=2, D=64, P=8, lens=lens, ragged=True)
    out, lse = call(T, which, d, cache, w.max_kv_len, **kw)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, 30, 2, bits), which)


@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_a_batch_without_nodes_or_without_a_prefix(which):
    T = U.require_gpu()
    w, d, cache, bits, kw = setup(which, 82, 0, 0, lens=[0, 0, 0])
    out, lse = call(T, which, d, cache, 0, **kw)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, 0, 0, bits), which)
    d["num_nodes"] = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = call(T, which, d, cache, 0, **kw, out=torch.full_like(out, 5.0))
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_window_and_4_bits_agree_where_4_bits_are_exact():
    """Values that the codes hold exactly: the same function by two kernels, and the values that
    the write says the cache holds are the ones that were written."""
    T = U.require_gpu()
    rng = np.random.default_rng(83)
    B, Hkv, D, P, n = 2, 2, 64, 16, 500
    levels = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float32)
    values = lambda: levels[rng.integers(0, 8, (B, n, Hkv, D))] * rng.choice(np.float32([-0.25, 0.25]), (B, n, Hkv, D))  # noqa: E731,E501
    rows = lambda: W.f32_to_bf16_bits(values())  # noqa: E731
    k, v = rows(), rows()
    k[..., ::32], v[..., ::32] = 0x3FC0, 0x3FC0              # 1.5, the top of every block
    w, d, _, _, _ = setup("window", 84, 0, 0, B=B, N=9, Hkv=Hkv, Hq=4, D=D, P=P, lens=[n, n])
    zeros = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    pool = len(w.k_cache)
    c4 = [zeros(pool, Hkv, P, D // 2), zeros(pool, Hkv, P, D // 2), zeros(pool, Hkv, P, 2, D // 32)]
    dk, dv = U.dev_bf16(k), U.dev_bf16(v)
    kh, vh = torch.empty_like(dk), torch.empty_like(dv)
    T.kv4_write(dk, dv, *c4, d["page_table"], torch.zeros(B, dtype=torch.int32, device="cuda"), k_held=kh, v_held=vh)
    assert same_all([kh, vh], [dk, dv])
    for b in range(B):
        pages, slots = torch.from_numpy(w.page_table[b, np.arange(n) // P]).long(), torch.arange(n) % P
        d["k_cache"][pages, slots], d["v_cache"][pages, slots] = dk[b], dv[b]
    for window, sinks in ((0, 0), (77, 3)):
        a, z = call(T, "window", d, [d["k_cache"], d["v_cache"]], n, window=window, sinks=sinks)
        c, y = call(T, "4 bits", d, c4, n, window=window, sinks=sinks)
        # the same scores up to the order of their fp32 sums; on either side a weight is off by
        # half a step of bf16, a part by half of one of fp16, a result by half a step of bf16
        top = max(1.5, float(d["v_tree"].abs().max()))
        assert (z - y).abs().max() <= 2.0 ** -12
        assert ((a.float() - c.float()).abs() <= 2 * top * (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -12)
                + 2.0 ** -7 * a.float().abs()).all()


def test_rows_of_other_sequences_and_pages_stay():
    """A padded batch: sequences that write nothing and pages that are nobody's, byte for byte."""
    T = U.require_gpu()
    rng = np.random.default_rng(85)
    B, rows, Hkv, D, P, pool = 4, 33, 3, 64, 8, 64
    fill = lambda *s: rng.integers(0, 256, size=s).astype(np.uint8)  # noqa: E731
    cache = [fill(pool, Hkv, P, D // 2), fill(pool, Hkv, P, D // 2), fill(pool, Hkv, P, 2, D // 32)]
    table = rng.permutation(pool)[:B * 8].reshape(B, 8).astype(np.int32)
    k, v = (W.f32_to_bf16_bits(rng.standard_normal((B, rows, Hkv, D), dtype=np.float32)) for _ in range(2))
    start, count = np.array([5, 31, 0, 7], np.int32), np.array([33, 0, 1, 32], np.int32)
    dc = [U.dev(a) for a in cache]
    T.kv4_write(U.dev_bf16(k), U.dev_bf16(v), *dc, U.dev(table), U.dev(start), count=U.dev(count))
    want = O.write4(k, v, *cache, table, start, count=count)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(dc, want))


@pytest.mark.parametrize("Hq,Hkv,N,D,lens", [
    (71, 1, 1, 128, [300, 5]),                   # one KV head, 71 rows
    (142, 2, 1, 64, [1300, 2000]),               # 71 rows, longer prefixes
    (13, 13, 1, 64, [100, 65]),                  # a row per KV head, an odd number of heads
    (21, 3, 5, 128, [77, 640]),                  # 35 rows
    (45, 5, 17, 64, [130, 700]),                 # 153 rows
    (2048, 1, 1, 64, [70, 3]),                   # the most rows by heads
    (1000, 2, 4, 128, [70, 300]),                # 2000 rows, blocks that end within a node
])
@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_head_layouts(which, Hq, Hkv, N, D, lens):
    T = U.require_gpu()
    w, d, cache, bits, kw = setup(which, 86, 50, 4, B=2, N=N, Hq=Hq, Hkv=Hkv, D=D, lens=lens, tree="forest")
    print(f"{which} Hq={Hq} Hkv={Hkv} N={N} D={D}", flush=True)
    out, lse = call(T, which, d, cache, w.max_kv_len, **kw)
    LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, 50, 4, bits), which)


def test_refusals():
    """Shapes, types, strides and devices that do not fit the call's other tensors."""
    T = U.require_gpu()
    w, d, cache, _, _ = setup("4 bits", 87)
    wd, dd, wcache, _, _ = setup("window", 87)

    def refused(match, which="4 bits", c=None, hint=900, **kw):
        args = dict(d if which == "4 bits" else dd)
        args.update({k: kw.pop(k) for k in list(kw) if k in args})
        with pytest.raises((ValueError, TypeError, RuntimeError), match=match):
            call(T, which, args, c or (cache if which == "4 bits" else wcache), hint, window=5, **kw)
    k4, v4, sc = cache
    refused("k4", c=[k4[..., :32], v4, sc])
    refused("v4", c=[k4, v4[:-1], sc])
    refused("scales", c=[k4, v4, sc[..., :2].contiguous()])
    refused("scales", c=[k4, v4, sc.to(torch.int32)])
    refused("k4", c=[k4.transpose(1, 2), v4, sc])            # the bf16 cache's order of heads and tokens
    refused("v_cache", "window", c=[wcache[0], wcache[1][:, ::2]])
    for which in ("window", "4 bits"):
        refused("q", which, q=d["q"].float())
        refused("k_tree", which, k_tree=d["k_tree"].cpu())
        refused("page_table", which, page_table=d["page_table"].long())
        refused("parent", which, parent=d["parent"][:, :-1])
        refused("kv_len", which, kv_len=d["kv_len"][:-1])
        refused("out", which, out=torch.empty_like(d["q"])[..., ::2])
        refused("lse", which, lse=torch.empty(d["q"].shape[:3], dtype=torch.bfloat16, device="cuda"))
        refused("workspace|WORKSPACE", which, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
        refused(".", which, hint=-1)
        refused(".", which, sinks=-1)
    k = torch.zeros((3, 4, 2, 128), dtype=torch.bfloat16, device="cuda")
    start = torch.zeros(3, dtype=torch.int32, device="cuda")

    def no_write(match, k=k, v=k, start=start, **kw):
        with pytest.raises((ValueError, TypeError, RuntimeError), match=match):
            T.kv4_write(k, v, *cache, d["page_table"], start, **kw)
    no_write("v", v=k[:, :3])
    no_write("k4", k=k[..., :64].contiguous(), v=k[..., :64].contiguous())
    no_write("start", start=start.long())
    no_write("idx", idx=torch.zeros((3, 3), dtype=torch.int32, device="cuda"))
    no_write("count", count=torch.zeros(2, dtype=torch.int32, device="cuda"))
    no_write("k_held", k_held=k[:, :2])
    no_write("overlap|OVERLAP", k_held=k, idx=torch.zeros((3, 4), dtype=torch.int32, device="cuda"))
    assert all(torch.equal(a, U.dev(b)) for a, b in zip(cache, LU.cache4(w)))


@pytest.mark.parametrize("N,Hq,Hkv,D", [(1, 8, 2, 128), (1, 1, 1, 64), (1, 32, 8, 128), (3, 40, 1, 128), (64, 8, 2, 64)])
@pytest.mark.parametrize("which", ["window", "4 bits"])
def test_a_window_that_begins_at_the_tile_behind_the_sinks(which, N, Hq, Hkv, D):
    """The last key before the window is the last one of the sinks' tile: no node sees it, also
    in a piece of work that has no tile of the tree, whose root paths are not looked up."""
    T = U.require_gpu()
    for window, sinks, n in ((4096, 4, 63), (1000, 1, 63), (2000, 65, 127), (2000, 65, 128), (640, 4, 62)):
        w, d, cache, bits, kw = setup(which, 88 + n, window, sinks, B=1, N=N, Hq=Hq, Hkv=Hkv, D=D, lens=[window + n],
                                      tree="chain")
        print(f"{which} N={N} window={window} sinks={sinks} len={window + n}", flush=True)
        zero = torch.zeros(1 << 22, device="cuda")
        zero.sort()                              # leaves zeros in many places of LDS
        out, lse = call(T, which, d, cache, w.max_kv_len, **kw)
        LU.check(w, U.bf16_to_f64(out), lse.cpu().numpy().astype(np.float64), LU.expected(w, window, sinks, bits), which)
