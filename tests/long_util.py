"""Inputs and bounds of the long-context operators' tests: batches inside a window whose
unseen positions hold NaN and whose unseen pages are given back, and caches in 4 bits."""
from __future__ import annotations

import numpy as np

from oracle import long_context as O
from paper_2602_21224_amd import workloads as W
from tests import cache_util as C


def workload(seed, *, B, N, Hq, Hkv, D, P, lens, window=0, sinks=0, tree="forest", ragged=False, depth=6):
    """Unseen slots (behind the window, past a prefix) are NaN in K and V; of pages without a
    visible position the table has -1, an id past the pool, or another sequence's page."""
    rng = np.random.default_rng(seed)

    def fn(r):
        n = int(r.integers(0, N + 1)) if ragged else N
        if n == 0:
            return np.zeros(0, np.int32)
        return {"capped": lambda: W.tree_random_depth_capped(r, n, depth), "forest": lambda: W.tree_uniform_forest(r, n),
                "chain": lambda: W.tree_chain(n)}[tree]()
    lens = np.asarray(lens, np.int32) if not isinstance(lens, tuple) else rng.integers(lens[0], lens[1] + 1, size=B)
    w = W.make_workload("long", seed, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, kv_len=lens, parent_fn=fn, V=8, P=P, poison=True,
                        with_logits=False)
    if window:
        pool = len(w.k_cache)
        for b, L in enumerate(w.kv_len):
            t = np.arange(L)
            unseen = t[(t >= sinks) & (t <= L - window)]
            pages = w.page_table[b, unseen // P]
            w.k_cache[pages, unseen % P] = W.BF16_NAN
            w.v_cache[pages, unseen % P] = W.BF16_NAN
            seen = np.setdiff1d(t, unseen) // P
            for page in np.setdiff1d(unseen // P, seen):
                w.page_table[b, page] = rng.choice([-1, pool, 0x7FFFFFFF, int(rng.integers(0, pool))])
    return w


def cache4(w):
    """(k4, v4, scales) of a workload's caches, rounded to 4 bits (NaN slots: NaN blocks)."""
    k4, ks = O.quantize4(w.k_cache.transpose(0, 2, 1, 3))
    v4, vs = O.quantize4(w.v_cache.transpose(0, 2, 1, 3))
    return k4, v4, np.ascontiguousarray(np.stack([ks, vs], axis=3))


def expected(w, window, sinks, cache=None, scale=0.0):
    """(out, lse, bound of |out error|, bound of |lse error|) in fp64. Scores are products
    summed in fp32; a weight is rounded once to bf16 (half a step, 2^-8), a split row's
    part to fp16 (2^-11), the output to bf16, and 2^-12 of the weights' sum of |v| is for
    the fp32 exponentials and sums."""
    k, v = (O.Rows16(w.k_cache), O.Rows16(w.v_cache)) if cache is None else (
        O.Rows4(cache[0], cache[2], 0), O.Rows4(cache[1], cache[2], 1))
    out, lse, mag = O.window_attention(w.q, w.k_tree, w.v_tree, k, v, w.page_table, w.kv_len, w.parent, window, sinks,
                                       num_nodes=w.num_nodes, scale=scale)
    norm = lambda x: np.sqrt(np.nanmax((W.bf16_bits_to_f32(x).astype(np.float64) ** 2).sum(-1), initial=0))  # noqa: E731
    qk = norm(w.q) * max(norm(w.k_tree), 1.25 * norm(w.k_cache)) * (scale if scale > 0 else w.D ** -0.5)
    with np.errstate(invalid="ignore"):
        bound = 2.0 ** -8 * (mag + np.abs(out)) + (2.0 ** -11 + 2.0 ** -12) * mag
        # weights follow the scores: each is off by as much, relatively, as its score absolutely
        bound += 2 * C.lse_bound(w.D, qk) * mag
        # fp16 ends: a part's row is scaled so that its largest value lies in [2^14, 2^15), and
        # what is below 2^-14 then is off by half of fp16's last step, 2^-25: at most 2^-39 of
        # that largest value, which is at most the largest |v|. The parts' weights sum to one.
        v = [np.nanmax(np.abs(W.bf16_bits_to_f32(x)), initial=0) for x in (w.v_tree, w.v_cache)]
        bound += 2.0 ** -39 * max(v[0], 1.25 * v[1])
        return out, lse, bound, C.lse_bound(w.D, qk) + 2.0 ** -21 * np.where(np.isfinite(lse), np.abs(lse), 0.0)


def check(w, got, z, want, label):
    """Compare (out fp64, lse) with expected()'s; padding rows are zeros and -inf."""
    out, lse, tol, ztol = want
    nodes = np.full(w.B, w.N) if w.num_nodes is None else w.num_nodes
    real = np.arange(w.N)[None, :] < nodes[:, None]
    assert (got[~real] == 0).all() and np.isneginf(z[~real]).all(), label
    err, zerr = np.abs(got - out)[real], np.abs(z[real] - lse[real])
    print(f"[{label}] max abs err {err.max(initial=0):.2e}, of its bound {(err / tol[real]).max(initial=0):.2f}; "
          f"lse {(zerr / ztol[real]).max(initial=0):.2f}", flush=True)
    assert np.isfinite(got[real]).all() and (err <= tol[real]).all(), label
    assert (zerr <= ztol[real]).all(), label
