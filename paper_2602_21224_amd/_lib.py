"""ctypes binding of libtreeverify (argument marshalling only).

Each wrapper takes torch tensors that already live on the GPU, checks dtype,
shape and contiguity, and passes raw device pointers plus the current HIP
stream to the C entry point of the same name. Every step of the computation
runs in the library's HIP kernels; there is no fallback of any kind: if the
library is missing or a call returns an error status, a Python exception is
raised.
"""
from __future__ import annotations

import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# TREEVERIFY_LIB names another build of the same library to load (the
# sanitizer test loads one whose host code carries AddressSanitizer and UBSan).
LIB_PATH = os.environ.get("TREEVERIFY_LIB") or os.path.join(HERE, "libtreeverify.so")

_lib = None


class TreeVerifyError(RuntimeError):
    pass


def load():
    """Load libtreeverify.so (built in-tree by `paper_2602_21224_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise TreeVerifyError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2602_21224_amd.build` (hipcc, gfx950)")
    lib = ctypes.CDLL(LIB_PATH)
    p, i, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.tv_abi_version.argtypes = []
    lib.tv_abi_version.restype = i
    lib.tv_status_string.argtypes = [i]
    lib.tv_status_string.restype = ctypes.c_char_p
    lib.tv_attention_workspace_size.argtypes = [i] * 5
    lib.tv_attention_workspace_size.restype = sz
    lib.tree_verify_attention.argtypes = [p] * 9 + [i] * 9 + [ctypes.c_float, p, p, p, sz, p]
    lib.tree_verify_attention.restype = i
    lib.tv_argmax_workspace_size.argtypes = [i] * 3
    lib.tv_argmax_workspace_size.restype = sz
    lib.tree_argmax_accept.argtypes = [p] * 4 + [i] * 3 + [p] * 5 + [sz, p]
    lib.tree_argmax_accept.restype = i
    lib.tree_argmax_accept_noalloc.argtypes = [p] * 4 + [i] * 3 + [p] * 5
    lib.tree_argmax_accept_noalloc.restype = i
    lib.kv_compact_accepted.argtypes = [p] * 8 + [i] * 7 + [p]
    lib.kv_compact_accepted.restype = i
    lib.tv_validate_inputs.argtypes = [p] * 4 + [i] * 5 + [p, p]
    lib.tv_validate_inputs.restype = i
    lib.tv_tree_build_workspace_size.argtypes = [i] * 5
    lib.tv_tree_build_workspace_size.restype = sz
    lib.tree_build.argtypes = [p] * 5 + [i] * 6 + [p] * 5 + [sz, p]
    lib.tree_build.restype = i
    lib.tree_resample.argtypes = [p] * 6 + [i] * 7 + [p] * 5 + [sz, p]
    lib.tree_resample.restype = i
    lib.tv_lm_head_workspace_size.argtypes = [i] * 4
    lib.tv_lm_head_workspace_size.restype = sz
    lib.tree_lm_head_argmax_accept.argtypes = [p] * 5 + [i] * 4 + [p] * 5 + [sz, p]
    lib.tree_lm_head_argmax_accept.restype = i
    lib.tv_shared_attention_workspace_size.argtypes = [i] * 6
    lib.tv_shared_attention_workspace_size.restype = sz
    lib.tree_verify_attention_shared.argtypes = ([p] * 11 + [i] * 10 + [ctypes.c_float, p, p, p, sz,
                                                                        p])
    lib.tree_verify_attention_shared.restype = i
    lib.kv_accumulate_weights.argtypes = [p] * 10 + [i] * 9 + [ctypes.c_float, p, p, p]
    lib.kv_accumulate_weights.restype = i
    lib.tv_evict_workspace_size.argtypes = [i] * 4
    lib.tv_evict_workspace_size.restype = sz
    lib.kv_evict.argtypes = [p] * 8 + [i] * 9 + [p] * 4 + [sz, p]
    lib.kv_evict.restype = i
    _lib = lib
    return lib


def _check(status: int, what: str):
    if status != 0:
        msg = load().tv_status_string(status).decode()
        raise TreeVerifyError(f"{what}: status {status} ({msg})")


def _ptr(t):
    return None if t is None else t.data_ptr()


# The smallest calls are bound by this module's own time per call (a wrapper took
# 7-10 us beside the library's 4 per launch): the current stream's handle is
# taken without building a Stream object (0.1 against 2.7 us), and an argument
# that is as wanted passes one test.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(torch.cuda.current_device())
    return torch.cuda.current_stream().cuda_stream


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)
_F32 = (torch.float32,)
_I32 = (torch.int32,)
_U8 = (torch.uint8,)


def _want(t, name, dtypes, shape=None):
    if (type(t) is torch.Tensor and t.dtype in dtypes and t.is_cuda and t.is_contiguous()
            and (shape is None or t.shape == shape)):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def abi_version() -> int:
    return int(load().tv_abi_version())


def attention_workspace_size(B, N, Hq, Hkv, D) -> int:
    return int(load().tv_attention_workspace_size(B, N, Hq, Hkv, D))


def argmax_workspace_size(B, N, V) -> int:
    return int(load().tv_argmax_workspace_size(B, N, V))


def tree_verify_attention(q, k_tree, v_tree, k_cache, v_cache, page_table, kv_len, parent, *,
                          max_kv_len: int, num_nodes=None, scale: float = 0.0, out=None,
                          lse=None, want_lse: bool = True, workspace=None, stream=None):
    """Tree-masked attention of every node over its sequence's paged prefix and
    its own root path. `num_nodes` (int32 [B], optional) makes the batch ragged.
    Returns (out bf16 [B,N,Hq,D], lse fp32 [B,N,Hq] or None)."""
    B, N, Hq, D = q.shape
    Hkv = k_tree.shape[2]
    num_pages, P = k_cache.shape[0], k_cache.shape[1]
    max_pages = page_table.shape[1]
    _want(q, "q", _BF16)
    _want(k_tree, "k_tree", _BF16, (B, N, Hkv, D))
    _want(v_tree, "v_tree", _BF16, (B, N, Hkv, D))
    _want(k_cache, "k_cache", _BF16, (num_pages, P, Hkv, D))
    _want(v_cache, "v_cache", _BF16, (num_pages, P, Hkv, D))
    _want(page_table, "page_table", _I32, (B, max_pages))
    _want(kv_len, "kv_len", _I32, (B,))
    _want(parent, "parent", _I32, (B, N))
    if num_nodes is not None:
        _want(num_nodes, "num_nodes", _I32, (B,))
    if out is None:
        out = torch.empty((B, N, Hq, D), dtype=torch.bfloat16, device=q.device)
    _want(out, "out", _BF16, (B, N, Hq, D))
    if lse is None and want_lse:
        lse = torch.empty((B, N, Hq), dtype=torch.float32, device=q.device)
    if lse is not None:
        _want(lse, "lse", _F32, (B, N, Hq))
    if workspace is None:
        need = attention_workspace_size(B, N, Hq, Hkv, D)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    _want(workspace, "workspace", _U8)
    st = load().tree_verify_attention(
        _ptr(q), _ptr(k_tree), _ptr(v_tree), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
        _ptr(kv_len), _ptr(parent), _ptr(num_nodes), B, N, Hq, Hkv, D, P, max_pages, num_pages,
        int(max_kv_len),
        float(scale), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "tree_verify_attention")
    return out, lse


def tree_argmax_accept(logits, draft_tokens, parent, *, num_nodes=None, argmax_out=None,
                       accept_len=None, accept_idx=None, bonus_token=None, workspace=None,
                       stream=None):
    """Per-node argmax, greedy longest accepted path and bonus token.
    `num_nodes` (int32 [B], optional) makes the batch ragged.
    Returns (argmax [B,N], accept_len [B], accept_idx [B,N], bonus [B]) int32."""
    B, N, V = logits.shape
    dev = logits.device
    _want(logits, "logits", _F32)
    _want(draft_tokens, "draft_tokens", _I32, (B, N))
    _want(parent, "parent", _I32, (B, N))
    if num_nodes is not None:
        _want(num_nodes, "num_nodes", _I32, (B,))
    mk = lambda shape: torch.empty(shape, dtype=torch.int32, device=dev)
    argmax_out = mk((B, N)) if argmax_out is None else argmax_out
    accept_len = mk((B,)) if accept_len is None else accept_len
    accept_idx = mk((B, N)) if accept_idx is None else accept_idx
    bonus_token = mk((B,)) if bonus_token is None else bonus_token
    for t, n, s in ((argmax_out, "argmax_out", (B, N)), (accept_len, "accept_len", (B,)),
                    (accept_idx, "accept_idx", (B, N)), (bonus_token, "bonus_token", (B,))):
        _want(t, n, _I32, s)
    if workspace is None:
        need = argmax_workspace_size(B, N, V)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    _want(workspace, "workspace", _U8)
    st = load().tree_argmax_accept(
        _ptr(logits), _ptr(draft_tokens), _ptr(parent), _ptr(num_nodes), B, N, V, _ptr(argmax_out),
        _ptr(accept_len), _ptr(accept_idx), _ptr(bonus_token), _ptr(workspace),
        workspace.numel(), _stream(stream))
    _check(st, "tree_argmax_accept")
    return argmax_out, accept_len, accept_idx, bonus_token


def tree_argmax_accept_noalloc(logits, draft_tokens, parent, *, argmax_out, accept_len,
                               accept_idx, bonus_token, num_nodes=None, stream=None):
    """tree_argmax_accept with the library's static per-GPU scratch instead of a
    workspace: nothing is allocated, so every output tensor must be given.
    Calls that can overlap on one GPU race on that scratch."""
    B, N, V = logits.shape
    _want(logits, "logits", _F32)
    _want(draft_tokens, "draft_tokens", _I32, (B, N))
    _want(parent, "parent", _I32, (B, N))
    if num_nodes is not None:
        _want(num_nodes, "num_nodes", _I32, (B,))
    for t, n, s in ((argmax_out, "argmax_out", (B, N)), (accept_len, "accept_len", (B,)),
                    (accept_idx, "accept_idx", (B, N)), (bonus_token, "bonus_token", (B,))):
        _want(t, n, _I32, s)
    st = load().tree_argmax_accept_noalloc(
        _ptr(logits), _ptr(draft_tokens), _ptr(parent), _ptr(num_nodes), B, N, V,
        _ptr(argmax_out), _ptr(accept_len), _ptr(accept_idx), _ptr(bonus_token), _stream(stream))
    _check(st, "tree_argmax_accept_noalloc")
    return argmax_out, accept_len, accept_idx, bonus_token


def lm_head_workspace_size(B, N, V, d) -> int:
    return int(load().tv_lm_head_workspace_size(B, N, V, d))


def tree_lm_head_argmax_accept(hidden, w_head, draft_tokens, parent, *, num_nodes=None,
                               argmax_out=None, accept_len=None, accept_idx=None,
                               bonus_token=None, workspace=None, stream=None):
    """LM head fused with greedy verification: hidden [B,N,d] bf16 times
    w_head [V,d] bf16, per-node argmax of the product (never stored), then the
    acceptance of tree_argmax_accept.
    Returns (argmax [B,N], accept_len [B], accept_idx [B,N], bonus [B]) int32."""
    B, N, d = hidden.shape
    V = w_head.shape[0]
    dev = hidden.device
    _want(hidden, "hidden", _BF16)
    _want(w_head, "w_head", _BF16, (V, d))
    _want(draft_tokens, "draft_tokens", _I32, (B, N))
    _want(parent, "parent", _I32, (B, N))
    if num_nodes is not None:
        _want(num_nodes, "num_nodes", _I32, (B,))
    mk = lambda shape: torch.empty(shape, dtype=torch.int32, device=dev)
    argmax_out = mk((B, N)) if argmax_out is None else argmax_out
    accept_len = mk((B,)) if accept_len is None else accept_len
    accept_idx = mk((B, N)) if accept_idx is None else accept_idx
    bonus_token = mk((B,)) if bonus_token is None else bonus_token
    for t, n, s in ((argmax_out, "argmax_out", (B, N)), (accept_len, "accept_len", (B,)),
                    (accept_idx, "accept_idx", (B, N)), (bonus_token, "bonus_token", (B,))):
        _want(t, n, _I32, s)
    if workspace is None:
        need = lm_head_workspace_size(B, N, V, d)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    _want(workspace, "workspace", _U8)
    st = load().tree_lm_head_argmax_accept(
        _ptr(hidden), _ptr(w_head), _ptr(draft_tokens), _ptr(parent), _ptr(num_nodes), B, N, V,
        d, _ptr(argmax_out), _ptr(accept_len), _ptr(accept_idx), _ptr(bonus_token),
        _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "tree_lm_head_argmax_accept")
    return argmax_out, accept_len, accept_idx, bonus_token


def kv_compact_accepted(k_tree, v_tree, k_cache, v_cache, page_table, kv_len, accept_idx,
                        accept_len, *, stream=None):
    """Write the accepted path's K/V rows into the cache after each prefix (in place)."""
    B, N, Hkv, D = k_tree.shape
    num_pages, P = k_cache.shape[0], k_cache.shape[1]
    max_pages = page_table.shape[1]
    _want(k_tree, "k_tree", _BF16)
    _want(v_tree, "v_tree", _BF16, (B, N, Hkv, D))
    _want(k_cache, "k_cache", _BF16, (num_pages, P, Hkv, D))
    _want(v_cache, "v_cache", _BF16, (num_pages, P, Hkv, D))
    _want(page_table, "page_table", _I32, (B, max_pages))
    _want(kv_len, "kv_len", _I32, (B,))
    _want(accept_idx, "accept_idx", _I32, (B, N))
    _want(accept_len, "accept_len", _I32, (B,))
    st = load().kv_compact_accepted(
        _ptr(k_tree), _ptr(v_tree), _ptr(k_cache), _ptr(v_cache), _ptr(page_table), _ptr(kv_len),
        _ptr(accept_idx), _ptr(accept_len), B, N, Hkv, D, P, max_pages, num_pages,
        _stream(stream))
    _check(st, "kv_compact_accepted")
    return k_cache, v_cache


def _want_on(dev, t, name, dtypes, shape=None):
    """_want, and on the device (an index) of the call's first tensor."""
    if (type(t) is torch.Tensor and t.dtype in dtypes and t.get_device() == dev
            and t.is_contiguous() and (shape is None or t.shape == shape)):
        return
    _want(t, name, dtypes, shape)
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, expected cuda:{dev}")


def _size(x):
    """A bound or budget as the C entry points' int: ctypes passes the low 32 bits of any
    integer, which made a budget of 2^40 one of 0. No sequence has 2^31 tokens, so more than
    that is that; what is negative stays so and is refused there."""
    x = int(x)
    return x if 0 <= x <= 0x7FFFFFFF else -1 if x < 0 else 0x7FFFFFFF


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _own(dev, stream, shape, dtype):
    """A tensor of the wrapper's own for a call on `stream`: from that stream's memory, whose
    earlier uses the call is behind (the current stream's may still be running)."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


def _call(what, dev, stream, own, *args):
    """Call the C entry point on device `dev` (made current for the call where it is not)
    and on `stream`. `own`: results that the wrapper allocated for another stream than the
    current one, where the caller goes on with them: the caching allocator does not hand
    them out again before the current stream is done with them."""
    fn = getattr(_lib or load(), what)
    if dev != _current_device():
        with torch.cuda.device(dev):
            st = fn(*args, _stream(stream))
    elif stream is None and _raw_stream is not None:
        st = fn(*args, _raw_stream(dev))
    else:
        st = fn(*args, _stream(stream))
    if stream is not None:
        for t in own:
            t.record_stream(torch.cuda.current_stream(dev))
    if st != 0:
        _check(st, what)


def shared_attention_workspace_size(B, N, Hq, Hkv, D, groups) -> int:
    return int(load().tv_shared_attention_workspace_size(B, N, Hq, Hkv, D, groups))


def tree_verify_attention_shared(q, k_tree, v_tree, k_cache, v_cache, page_table, kv_len, parent,
                                 group_start, shared_len, *, max_kv_len: int, num_nodes=None,
                                 scale: float = 0.0, out=None, lse=None, want_lse: bool = True,
                                 workspace=None, stream=None):
    """tree_verify_attention for a batch whose sequences share prefixes: sequences
    group_start[s] .. group_start[s+1]-1 hold their first shared_len[s] tokens in the
    same pages, and those rows are read once for the whole group, where that can pay
    (not with as many groups as sequences, empty ones among them). group_start
    [groups + 1] and shared_len [groups] are int32 (both None: no groups).
    Returns (out bf16 [B,N,Hq,D], lse fp32 [B,N,Hq] or None)."""
    B, N, Hq, D = q.shape
    Hkv = k_tree.shape[2]
    num_pages, P = k_cache.shape[0], k_cache.shape[1]
    max_pages = page_table.shape[1]
    dev = q.get_device()
    _want(q, "q", _BF16)
    _want_on(dev, k_tree, "k_tree", _BF16, (B, N, Hkv, D))
    _want_on(dev, v_tree, "v_tree", _BF16, (B, N, Hkv, D))
    _want_on(dev, k_cache, "k_cache", _BF16, (num_pages, P, Hkv, D))
    _want_on(dev, v_cache, "v_cache", _BF16, (num_pages, P, Hkv, D))
    _want_on(dev, page_table, "page_table", _I32, (B, max_pages))
    _want_on(dev, kv_len, "kv_len", _I32, (B,))
    _want_on(dev, parent, "parent", _I32, (B, N))
    if num_nodes is not None:
        _want_on(dev, num_nodes, "num_nodes", _I32, (B,))
    if (group_start is None) != (shared_len is None):
        raise ValueError("group_start and shared_len are given together")
    groups = 0 if shared_len is None else shared_len.shape[0]
    if groups > 0:
        _want_on(dev, group_start, "group_start", _I32, (groups + 1,))
        _want_on(dev, shared_len, "shared_len", _I32, (groups,))
    own = []
    if out is None:
        out = _own(dev, stream, (B, N, Hq, D), torch.bfloat16)
        own.append(out)
    _want_on(dev, out, "out", _BF16, (B, N, Hq, D))
    if lse is None and want_lse:
        lse = _own(dev, stream, (B, N, Hq), torch.float32)
        own.append(lse)
    if lse is not None:
        _want_on(dev, lse, "lse", _F32, (B, N, Hq))
    if workspace is None:
        need = shared_attention_workspace_size(B, N, Hq, Hkv, D, groups)
        workspace = _own(dev, stream, max(need, 16), torch.uint8)
    _want_on(dev, workspace, "workspace", _U8)
    _call("tree_verify_attention_shared", dev, stream, own,
          _ptr(q), _ptr(k_tree), _ptr(v_tree), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
          _ptr(kv_len), _ptr(parent), _ptr(num_nodes), _ptr(group_start if groups else None),
          _ptr(shared_len if groups else None), groups, B, N, Hq, Hkv, D, P, max_pages, num_pages,
          _size(max_kv_len), float(scale), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel())
    return out, lse


def kv_accumulate_weights(q, lse, k_cache, page_table, kv_len, accept_idx, accept_len, weight,
                          position, seen, *, max_kv_len: int, fixed_len=None, weight_out=None,
                          scale: float = 0.0, stream=None):
    """Add the attention weight that the accepted path's query rows gave every cached
    key to `weight` [B, Hkv, max_pages * P] fp32, and enter the path's own keys (weight
    and `position`, int32 of the same shape). Call it between kv_compact_accepted and
    advancing kv_len and `seen` [B]. Updates `weight` unless `weight_out` is given, and
    `position`. Returns (weight_out, position)."""
    B, N, Hq, D = q.shape
    num_pages, P, Hkv = k_cache.shape[0], k_cache.shape[1], k_cache.shape[2]
    max_pages = page_table.shape[1]
    dev = q.get_device()
    slots = (B, Hkv, max_pages * P)
    _want(q, "q", _BF16)
    _want_on(dev, lse, "lse", _F32, (B, N, Hq))
    _want_on(dev, k_cache, "k_cache", _BF16, (num_pages, P, Hkv, D))
    _want_on(dev, page_table, "page_table", _I32, (B, max_pages))
    _want_on(dev, kv_len, "kv_len", _I32, (B,))
    _want_on(dev, accept_idx, "accept_idx", _I32, (B, N))
    _want_on(dev, accept_len, "accept_len", _I32, (B,))
    _want_on(dev, weight, "weight", _F32, slots)
    _want_on(dev, position, "position", _I32, slots)
    _want_on(dev, seen, "seen", _I32, (B,))
    if fixed_len is not None:
        _want_on(dev, fixed_len, "fixed_len", _I32, (B,))
    if weight_out is None:
        weight_out = weight
    _want_on(dev, weight_out, "weight_out", _F32, slots)
    _call("kv_accumulate_weights", dev, stream, (),
          _ptr(q), _ptr(lse), _ptr(k_cache), _ptr(page_table), _ptr(kv_len), _ptr(accept_idx),
          _ptr(accept_len), _ptr(seen), _ptr(fixed_len), _ptr(weight), B, N, Hq, Hkv, D, P,
          max_pages, num_pages, _size(max_kv_len), float(scale), _ptr(weight_out), _ptr(position))
    return weight_out, position


def evict_workspace_size(B, Hkv, max_pages, P) -> int:
    return int(load().tv_evict_workspace_size(B, Hkv, max_pages, P))


def kv_evict(weight, position, k_cache, v_cache, page_table, kv_len, seen, *, max_kv_len: int,
             budget: int, recent: int = 0, fixed_len=None, weight_out=None, position_out=None,
             kept_len=None, workspace=None, stream=None):
    """Cut every sequence's cache to max(budget, fixed_len) slots per KV head: the fixed
    ones, those of the `recent` newest positions, then the heaviest. The kept rows past
    that length move into the evicted slots below it (K, V, weight, position). Updates
    the caches, and `weight` and `position` unless other arrays are given for them.
    `kept_len` may not overlap kv_len, seen or fixed_len.
    Returns (weight_out, position_out, kept_len)."""
    num_pages, P, Hkv, D = k_cache.shape
    B, max_pages = page_table.shape
    dev = k_cache.get_device()
    slots = (B, Hkv, max_pages * P)
    _want(k_cache, "k_cache", _BF16)
    _want_on(dev, v_cache, "v_cache", _BF16, (num_pages, P, Hkv, D))
    _want_on(dev, page_table, "page_table", _I32, (B, max_pages))
    _want_on(dev, weight, "weight", _F32, slots)
    _want_on(dev, position, "position", _I32, slots)
    _want_on(dev, kv_len, "kv_len", _I32, (B,))
    _want_on(dev, seen, "seen", _I32, (B,))
    if fixed_len is not None:
        _want_on(dev, fixed_len, "fixed_len", _I32, (B,))
    if weight_out is None:
        weight_out = weight
    if position_out is None:
        position_out = position
    _want_on(dev, weight_out, "weight_out", _F32, slots)
    _want_on(dev, position_out, "position_out", _I32, slots)
    own = []
    if kept_len is None:
        kept_len = _own(dev, stream, (B,), torch.int32)
        own.append(kept_len)
    _want_on(dev, kept_len, "kept_len", _I32, (B,))
    if kept_len.data_ptr() == kv_len.data_ptr() and B > 0:
        raise ValueError("kept_len must not be kv_len itself")
    if workspace is None:
        need = evict_workspace_size(B, Hkv, max_pages, P)
        workspace = _own(dev, stream, max(need, 16), torch.uint8)
    _want_on(dev, workspace, "workspace", _U8)
    _call("kv_evict", dev, stream, own,
          _ptr(weight), _ptr(position), _ptr(k_cache), _ptr(v_cache), _ptr(page_table),
          _ptr(kv_len), _ptr(seen), _ptr(fixed_len), B, Hkv, D, P, max_pages, num_pages,
          _size(max_kv_len), _size(budget), _size(recent), _ptr(weight_out), _ptr(position_out),
          _ptr(kept_len), _ptr(workspace), workspace.numel())
    return weight_out, position_out, kept_len


def tv_validate_inputs(page_table, kv_len, parent, *, P: int, num_pages: int, num_nodes=None,
                       stream=None):
    """Device-side contract check; returns the status bit set as a 1-element int32 tensor."""
    B, N = parent.shape
    max_pages = page_table.shape[1]
    _want(page_table, "page_table", _I32, (B, max_pages))
    _want(kv_len, "kv_len", _I32, (B,))
    _want(parent, "parent", _I32, (B, N))
    if num_nodes is not None:
        _want(num_nodes, "num_nodes", _I32, (B,))
    word = torch.empty(1, dtype=torch.int32, device=parent.device)
    st = load().tv_validate_inputs(_ptr(page_table), _ptr(kv_len), _ptr(parent), _ptr(num_nodes), B, N, P,
                                   max_pages, num_pages, _ptr(word), _stream(stream))
    _check(st, "tv_validate_inputs")
    return word


def tree_build_workspace_size(B, S, V, H, k) -> int:
    return int(load().tv_tree_build_workspace_size(B, S, V, H, k))


def tree_build(logits, root_token, token_info, hot_vocab, hot_index, *, k: int, budget: int,
               parent=None, token=None, joint=None, num_nodes=None, workspace=None, stream=None):
    """Draft tree by token-info sampling (Alg. 1) pruned to `budget` nodes (§5.2).

    logits [B, S, V] fp32, root_token [B] int32, token_info [H, H] bf16 (or
    None with H = 0), hot_vocab [H] and hot_index [V] int32. Returns (parent,
    token, joint, num_nodes): [B, budget] int32, int32, fp32 and [B] int32.
    """
    B, S, V = logits.shape
    _want(logits, "logits", _F32)
    _want(root_token, "root_token", _I32, (B,))
    H = 0 if token_info is None else token_info.shape[0]
    if H > 0:
        _want(token_info, "token_info", _BF16, (H, H))
        _want(hot_vocab, "hot_vocab", _I32, (H,))
        _want(hot_index, "hot_index", _I32, (V,))
    dev = logits.device
    mk = lambda shape, dt: torch.empty(shape, dtype=dt, device=dev)
    parent = mk((B, budget), torch.int32) if parent is None else parent
    token = mk((B, budget), torch.int32) if token is None else token
    joint = mk((B, budget), torch.float32) if joint is None else joint
    num_nodes = mk((B,), torch.int32) if num_nodes is None else num_nodes
    _want(parent, "parent", _I32, (B, budget))
    _want(token, "token", _I32, (B, budget))
    _want(joint, "joint", _F32, (B, budget))
    _want(num_nodes, "num_nodes", _I32, (B,))
    need = tree_build_workspace_size(B, S, V, H, k)
    if need == 0:
        raise TreeVerifyError(f"tree_build: unsupported shape B={B} S={S} V={V} H={H} k={k}")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    st = load().tree_build(
        _ptr(logits), _ptr(root_token), _ptr(token_info if H > 0 else None),
        _ptr(hot_vocab if H > 0 else None), _ptr(hot_index if H > 0 else None), B, S, V, H, k,
        budget, _ptr(parent), _ptr(token), _ptr(joint), _ptr(num_nodes), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "tree_build")
    return parent, token, joint, num_nodes


def tree_resample(logits, bonus_token, accept_len, token_info, hot_vocab, hot_index, *, k: int,
                  r: int, budget: int, parent=None, token=None, joint=None, num_nodes=None,
                  workspace=None, stream=None):
    """Re-sampled draft trees after verification (Alg. 2): rooted at the bonus
    tokens, drawn from logits rows accept_len .. S-1 when more than r remain.
    Same tensors and outputs as tree_build, plus bonus_token / accept_len [B]."""
    B, S, V = logits.shape
    _want(logits, "logits", _F32)
    _want(bonus_token, "bonus_token", _I32, (B,))
    _want(accept_len, "accept_len", _I32, (B,))
    H = 0 if token_info is None else token_info.shape[0]
    if H > 0:
        _want(token_info, "token_info", _BF16, (H, H))
        _want(hot_vocab, "hot_vocab", _I32, (H,))
        _want(hot_index, "hot_index", _I32, (V,))
    dev = logits.device
    mk = lambda shape, dt: torch.empty(shape, dtype=dt, device=dev)
    parent = mk((B, budget), torch.int32) if parent is None else parent
    token = mk((B, budget), torch.int32) if token is None else token
    joint = mk((B, budget), torch.float32) if joint is None else joint
    num_nodes = mk((B,), torch.int32) if num_nodes is None else num_nodes
    _want(parent, "parent", _I32, (B, budget))
    _want(token, "token", _I32, (B, budget))
    _want(joint, "joint", _F32, (B, budget))
    _want(num_nodes, "num_nodes", _I32, (B,))
    need = tree_build_workspace_size(B, S, V, H, k)
    if need == 0:
        raise TreeVerifyError(f"tree_resample: unsupported shape B={B} S={S} V={V} H={H} k={k}")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    st = load().tree_resample(
        _ptr(logits), _ptr(bonus_token), _ptr(accept_len), _ptr(token_info if H > 0 else None),
        _ptr(hot_vocab if H > 0 else None), _ptr(hot_index if H > 0 else None), B, S, V, H, k, r,
        budget, _ptr(parent), _ptr(token), _ptr(joint), _ptr(num_nodes), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "tree_resample")
    return parent, token, joint, num_nodes

