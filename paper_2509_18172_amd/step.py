"""The operators between the products of a step, on torch tensors: the plan of
a batch, the paged key/value cache, attention for trees of drafted tokens, the
norms around a block and the adjustment of logits (include/sbvr.h says what
each computes).  Marshalling only, as the package's other helpers: shapes are
checked here, outputs come from torch, and a non-zero status raises
``SBVRError``.

A step in order: ``batch_plan`` (pages, slots, masks), per layer
``residual_norm`` -> products -> ``cache_write`` -> ``tree_attention`` ->
products, and ``adjust_logits`` on the last product.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import (SBVR_BF16, SBVR_F16, SBVR_F32, CacheStruct, LogitsStruct, SBVRError, _lib, _stream,
               sbvr_tree_attention_workspace_bytes)

# These calls are short, and one step makes hundreds of them: the library's
# functions are called without the wrappers of the same names.
_empty = torch.empty_strided  # (half of torch.empty's time)
_workspace_bytes = functools.lru_cache(maxsize=256)(sbvr_tree_attention_workspace_bytes)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _on(stream, device) -> int:
    """The handle of `stream`, by default the current stream of `device`."""
    return _stream(stream) if stream is not None or _raw_stream is None else _raw_stream(device.index)


def _check(status: int, what: str):
    if status:
        raise SBVRError(status, what)


_DTYPE = {torch.float16: SBVR_F16, torch.bfloat16: SBVR_BF16, torch.float32: SBVR_F32}


def _dense(t, dtype, shape, device, what):
    """The pointer of an optional contiguous tensor of one dtype and shape."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise AssertionError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _list(t, dtype, device, what):
    """The pointer and length of an optional contiguous 1-D tensor."""
    if t is None:
        return None, 0
    n, = t.shape
    return _dense(t, dtype, (n,), device, what), n


def _rows(t, dtype, shape, device, what):
    """The pointer and row stride of a 2-D tensor with contiguous rows."""
    if t.dtype != dtype or t.shape != shape or t.device != device or (t.stride(1) != 1 and shape[1] != 1):
        raise AssertionError(f"{what} must be a {dtype} tensor {tuple(shape)} of contiguous rows on {device}")
    return t.data_ptr(), t.stride(0)


def _table(page_table, R, device):
    rows, pages = page_table.shape
    pointer, stride = _rows(page_table, torch.int32, (R, pages), device, "page_table")
    # a single row's stride means nothing, and torch may report a smaller one
    return pointer, pages, max(stride, pages)


class BatchPlan:
    """What ``batch_plan`` returns: device tensors query_start int32 [R + 1],
    token_request and positions int32 [T], slots int64 [T], tree_mask int64
    [T] (bits of a uint64), used int32 [2] (pages taken, new tokens)."""

    def __init__(self, R: int, T: int, device):
        self.query_start = _empty((R + 1,), (1,), dtype=torch.int32, device=device)
        self.token_request = _empty((T,), (1,), dtype=torch.int32, device=device)
        self.positions = torch.empty_like(self.token_request)
        self.slots = _empty((T,), (1,), dtype=torch.int64, device=device)
        self.tree_mask = torch.empty_like(self.slots)
        self.used = _empty((2,), (1,), dtype=torch.int32, device=device)


def batch_plan(context_lens, new_lens, free_pages, page_table, page_size: int, n_tokens: int, parents=None, out=None,
               stream=None) -> BatchPlan:
    """Pages for a step's new tokens (entered into page_table, in place) and
    what the other operators need per token.  context_lens, new_lens int32
    [R]; free_pages int32 [n]; page_table int32 [R][max_pages]; parents int32
    [n_tokens] within each request (None: chains); n_tokens: room for the
    step's tokens.  out: a BatchPlan of the same sizes to fill."""
    device = context_lens.device
    assert context_lens.is_cuda and context_lens.dim() == 1
    R, T = context_lens.shape[0], int(n_tokens)
    i32 = torch.int32
    table, max_pages, stride = _table(page_table, R, device)
    if out is None:
        p = BatchPlan(R, T, device)
    else:
        p = out
        for name, dtype, n in (("query_start", i32, R + 1), ("token_request", i32, T), ("positions", i32, T),
                               ("slots", torch.int64, T), ("tree_mask", torch.int64, T), ("used", i32, 2)):
            _dense(getattr(p, name), dtype, (n,), device, name)
    _check(_lib.sbvr_batch_plan(R, T, page_size, _dense(context_lens, i32, (R,), device, "context_lens"),
                           _dense(new_lens, i32, (R,), device, "new_lens"),
                           *_list(free_pages, i32, device, "free_pages"),
                           _dense(parents, i32, (T,), device, "parents"), table, max_pages, stride,
                           p.query_start.data_ptr(), p.token_request.data_ptr(), p.positions.data_ptr(),
                           p.slots.data_ptr(), p.tree_mask.data_ptr(), p.used.data_ptr(), _on(stream, device)),
           "sbvr_batch_plan")
    return p


class KVCache:
    """A paged key/value cache: two fp16 or bf16 tensors [pages][page_size]
    [kv_heads][head_dim], of any strides with contiguous heads (a head-major
    page is a transposed view)."""

    def __init__(self, k, v):
        n_pages, page_size, heads, dim = k.shape
        ks, vs = k.stride(), v.stride()
        assert k.shape == v.shape and k.dtype == v.dtype and k.dtype in _DTYPE and k.is_cuda and k.device == v.device, \
            "k and v must be alike, [pages][page_size][kv_heads][head_dim]"
        assert ks[3] == 1 and vs[3] == 1, "a head's elements must be contiguous"
        self.k, self.v = k, v
        self.dtype, self.device, self.kv_heads, self.head_dim = k.dtype, k.device, heads, dim
        # (the struct is kept with its address, which the library reads it at)
        self.struct = CacheStruct(k.data_ptr(), v.data_ptr(), *ks[:3], *vs[:3], n_pages, page_size, heads, dim,
                                  _DTYPE[k.dtype])
        self.address = C.addressof(self.struct)

    @staticmethod
    def alloc(n_pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.float16, device="cuda"):
        shape = (n_pages, page_size, kv_heads, head_dim)
        return KVCache(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))


def _heads(t, heads, dim, cache, what):
    """The pointer and the token and head strides of a [T][heads][dim] tensor
    that goes with a cache."""
    token, head, one = t.stride()
    if t.shape[1:] != (heads, dim) or one != 1 or t.dtype != cache.dtype or t.device != cache.device:
        raise AssertionError(f"{what} must be a {cache.dtype} tensor [tokens][{heads}][{dim}] with contiguous heads on "
                             "the cache's device")
    return t.data_ptr(), token, head


def cache_write(cache: KVCache, k, v, slots, stream=None):
    """Write a step's keys and values [T][kv_heads][head_dim] (views with
    contiguous heads) to the slots (int64 [T]; negative: skipped)."""
    heads, dim = cache.kv_heads, cache.head_dim
    T = k.shape[0]
    assert v.shape[0] == T, "k and v must have the same tokens"
    _check(_lib.sbvr_cache_write(cache.address, T, *_heads(k, heads, dim, cache, "k"), *_heads(v, heads, dim, cache, "v"),
                            _dense(slots, torch.int64, (T,), cache.device, "slots"), _on(stream, cache.device)),
           "sbvr_cache_write")


def tree_attention(q, cache: KVCache, page_table, context_lens, query_start, tree_mask, max_new: int, scale=None,
                   out=None, workspace=None, stream=None):
    """Attention of a step's tokens q [T][heads][head_dim] over the cache,
    which already holds their keys and values; max_new: the most new tokens of
    a request; scale: 1 / sqrt(head_dim) by default.  Returns [T][heads]
    [head_dim].  workspace: a uint8 tensor of
    sbvr_tree_attention_workspace_bytes, by default a new one."""
    T, H, D = q.shape
    R, device = context_lens.shape[0], cache.device
    qp, q_token, q_head = _heads(q, H, cache.head_dim, cache, "q")
    table, max_pages, stride = _table(page_table, R, device)
    if out is None:
        out = _empty((T, H, D), (H * D, D, 1), dtype=q.dtype, device=device)
    need = _workspace_bytes(R, max_new, H, cache.kv_heads, D)
    if workspace is None and need:
        workspace = _empty((need,), (1,), dtype=torch.uint8, device=device)
        if stream is not None:
            workspace.record_stream(stream)
    _check(_lib.sbvr_tree_attention(cache.address, R, T, H, qp, q_token, q_head, table, max_pages, stride,
                               _dense(context_lens, torch.int32, (R,), device, "context_lens"),
                               _dense(query_start, torch.int32, (R + 1,), device, "query_start"),
                               _dense(tree_mask, torch.int64, (T,), device, "tree_mask"), max_new,
                               float(D ** -0.5 if scale is None else scale),
                               _dense(out, q.dtype, (T, H, D), device, "out"),
                               *_list(workspace, torch.uint8, device, "workspace"), _on(stream, device)),
           "sbvr_tree_attention")
    return out


def residual_norm(x, y=None, post_weight=None, gate=None, scale: float = 1.0, pre_weight=None, eps: float = 1e-5,
                  x_out=None, h_out=None, stream=None):
    """x' = x + scale * gate * rms(y) * post_weight and h = rms(x') *
    pre_weight for tokens x [T][H] (fp16, bf16 or fp32 stream), y [T][H] and
    gate [T][H] or [H] (fp16 or bf16); returns (x', h).  Without pre_weight h
    is None; without y x' is x itself.  x_out may be x."""
    T, H = x.shape
    device = x.device
    dtype = (y if y is not None else pre_weight if pre_weight is not None else x).dtype
    assert x.is_cuda and x.dtype in _DTYPE and dtype in _DTYPE, "x must be a GPU tensor of fp16, bf16 or fp32"
    xp, x_stride = _rows(x, x.dtype, (T, H), device, "x")
    op, o_stride, hp, h_stride, yp, y_stride, gp, g_stride = None, 0, None, 0, None, 0, None, 0
    if y is None:
        assert post_weight is None and gate is None and x_out is None, \
            "post_weight, gate and x_out need a y"
        assert pre_weight is not None, "nothing to compute: neither y nor pre_weight"
    else:
        yp, y_stride = _rows(y, dtype, (T, H), device, "y")
        if gate is not None:
            if gate.dim() == 1:
                gp = _dense(gate, dtype, (H,), device, "gate")
            else:
                gp, g_stride = _rows(gate, dtype, (T, H), device, "gate")
        if x_out is None:
            x_out = _empty((T, H), (H, 1), dtype=x.dtype, device=device)
        op, o_stride = _rows(x_out, x.dtype, (T, H), device, "x_out")
    if pre_weight is None:
        assert h_out is None, "an h needs a pre_weight"
    else:
        if h_out is None:
            h_out = _empty((T, H), (H, 1), dtype=dtype, device=device)
        hp, h_stride = _rows(h_out, dtype, (T, H), device, "h_out")
    _check(_lib.sbvr_residual_norm(T, H, _DTYPE[dtype], _DTYPE[x.dtype], xp, x_stride, yp, y_stride,
                              _dense(post_weight, dtype, (H,), device, "post_weight"), gp, g_stride, float(scale),
                              _dense(pre_weight, dtype, (H,), device, "pre_weight"), float(eps), op, o_stride, hp,
                              h_stride, _on(stream, device)), "sbvr_residual_norm")
    return (x if y is None else x_out), h_out


def adjust_logits(logits, history=None, history_start=None, prompt_lens=None, repetition=None, frequency=None,
                  presence=None, temperature=None, bias_tokens=None, bias_values=None, bias_start=None, grammar=None,
                  grammar_rows=None, token_request=None, query_start=None, tree_mask=None, draft_tokens=None,
                  n_requests=None, out=None, out_dtype=None, stream=None):
    """The logits [T][V] (fp16, bf16 or fp32) with the penalties, biases,
    temperatures and grammar masks of their requests applied (every part
    optional); out may be logits.  The number of requests R comes from
    history_start, bias_start or the parameters per request, or n_requests;
    without token_request row t is request t."""
    assert logits.dim() == 2 and logits.is_cuda and logits.dtype in _DTYPE
    T, V = logits.shape
    device = logits.device
    i32, f32 = torch.int32, torch.float32
    R = n_requests
    if R is None:
        for per_request in (prompt_lens, repetition, frequency, presence, temperature):
            if per_request is not None:
                R = per_request.shape[0]
                break
        else:
            starts = history_start if history_start is not None else bias_start if bias_start is not None else query_start
            R = T if starts is None else starts.shape[0] - 1
    if out is None:
        out = _empty((T, V), (V, 1), dtype=out_dtype or logits.dtype, device=device)
    assert out.dtype in _DTYPE and (out_dtype is None or out.dtype == out_dtype)
    assert (history is None) == (history_start is None), "history and history_start go together"
    assert (bias_tokens is None) == (bias_start is None) == (bias_values is None), "the three bias tensors go together"
    lp, l_stride = _rows(logits, logits.dtype, (T, V), device, "logits")
    op, o_stride = _rows(out, out.dtype, (T, V), device, "out")
    n_bias = 0 if bias_tokens is None else bias_tokens.shape[0]
    gp, g_stride, g_count = None, 0, 0
    if grammar is not None:
        g_count = grammar.shape[0]
        gp, g_stride = _rows(grammar, i32, (g_count, (V + 31) // 32), device, "grammar")
        g_stride = max(g_stride, grammar.shape[1])
    args = LogitsStruct(R, T, V, _DTYPE[logits.dtype], _DTYPE[out.dtype], lp, l_stride, op, o_stride,
                        _dense(token_request, i32, (T,), device, "token_request"),
                        _list(history, i32, device, "history")[0],
                        _dense(history_start, i32, (R + 1,), device, "history_start"),
                        _dense(prompt_lens, i32, (R,), device, "prompt_lens"),
                        _dense(repetition, f32, (R,), device, "repetition"),
                        _dense(frequency, f32, (R,), device, "frequency"),
                        _dense(presence, f32, (R,), device, "presence"),
                        _dense(temperature, f32, (R,), device, "temperature"),
                        _dense(bias_tokens, i32, (n_bias,), device, "bias_tokens"),
                        _dense(bias_start, i32, (R + 1,), device, "bias_start"),
                        _dense(bias_values, f32, (n_bias,), device, "bias_values"), gp, g_stride,
                        _dense(grammar_rows, i32, (T,), device, "grammar_rows"), g_count,
                        _dense(draft_tokens, i32, (T,), device, "draft_tokens"),
                        _dense(query_start, i32, (R + 1,), device, "query_start"),
                        _dense(tree_mask, torch.int64, (T,), device, "tree_mask"))
    _check(_lib.sbvr_adjust_logits(C.addressof(args), _on(stream, device)), "sbvr_adjust_logits")
    return out
