"""The operators between the products of a step, on torch tensors: the plan of
a batch, the paged key/value cache, attention for trees of drafted tokens, the
norms around a block and the adjustment of logits (include/sbvr.h says what
each computes).  Marshalling only, as the package's other helpers: shapes are
checked (AssertionError), outputs come from torch, and a non-zero status raises
``SBVRError``.  The helpers themselves are native (csrc/step_bind.cpp).

A step in order: ``batch_plan`` (pages, slots, masks), per layer
``residual_norm`` -> products -> ``cache_write`` -> ``tree_attention`` ->
products, and ``adjust_logits`` on the last product.  ``stream``: a
torch.cuda.Stream of the tensors' device, by default its current one; the call
is made with that device and stream as the current ones, so outputs and
workspaces belong to the stream as they do under ``torch.cuda.stream(stream)``.

Forward only: results carry no gradient, whatever the inputs say, and what is
written in place (page_table, a cache, x_out, out) is not marked as changed.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os

import torch

from . import SBVRError, _lib
from .build import binding_path


def _load():
    path = binding_path()
    if not os.path.exists(path):
        raise ImportError(f"SBVR tensor binding not built ({path}); run "
                          "`python -c 'import __graft_entry__ as g; g.build()'`")
    loader = importlib.machinery.ExtensionFileLoader("_sbvr_step", path)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_sbvr_step", loader))
    loader.exec_module(module)
    return module


_native = _load()

FUNCTIONS = ("sbvr_batch_plan", "sbvr_cache_write", "sbvr_tree_attention_workspace_bytes", "sbvr_tree_attention",
             "sbvr_tree_attention_whole", "sbvr_residual_norm", "sbvr_adjust_logits")


def _exchange_device(index: int) -> int:
    before = torch.cuda.current_device()
    torch.cuda.set_device(index)
    return before


def _connect():
    """Hands the binding the library's functions and what it asks of torch
    (the raw forms spare objects of streams and devices)."""
    stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda index: torch.cuda.current_stream(index).cuda_stream)
    device = getattr(torch._C, "_cuda_exchangeDevice", None) or _exchange_device
    _native.connect({n: C.cast(getattr(_lib, n), C.c_void_p).value for n in FUNCTIONS}, SBVRError, stream, device)


_connect()


class BatchPlan:
    """What ``batch_plan`` returns: device tensors query_start int32 [R + 1],
    token_request and positions int32 [T], slots int64 [T], tree_mask int64
    [T] (bits of a uint64), used int32 [2] (pages taken, new tokens)."""
    __slots__ = ("query_start", "token_request", "positions", "slots", "tree_mask", "used")

    def __init__(self, query_start, token_request, positions, slots, tree_mask, used):
        self.query_start, self.token_request, self.positions = query_start, token_request, positions
        self.slots, self.tree_mask, self.used = slots, tree_mask, used


def batch_plan(context_lens, new_lens, free_pages, page_table, page_size: int, n_tokens: int, parents=None, out=None,
               stream=None) -> BatchPlan:
    """Pages for a step's new tokens (entered into page_table, in place) and
    what the other operators need per token.  context_lens, new_lens int32
    [R]; free_pages int32 [n]; page_table int32 [R][max_pages]; parents int32
    [n_tokens] within each request (None: chains); n_tokens: room for the
    step's tokens.  out: a BatchPlan of the same sizes to fill."""
    if out is None:
        return BatchPlan(*_native.batch_plan(context_lens, new_lens, free_pages, page_table, page_size, n_tokens, parents,
                                             None, stream))
    _native.batch_plan(context_lens, new_lens, free_pages, page_table, page_size, n_tokens, parents,
                       [getattr(out, name) for name in BatchPlan.__slots__], stream)
    return out


class KVCache:
    """A paged key/value cache: two fp16 or bf16 tensors [pages][page_size]
    [kv_heads][head_dim], of any strides with contiguous heads (a head-major
    page is a transposed view)."""
    __slots__ = ("k", "v")

    def __init__(self, k, v):
        self.k, self.v = k, v

    @staticmethod
    def alloc(n_pages: int, page_size: int, kv_heads: int, head_dim: int, dtype=torch.float16, device="cuda"):
        shape = (n_pages, page_size, kv_heads, head_dim)
        return KVCache(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device))


def cache_write(cache: KVCache, k, v, slots, stream=None):
    """Write a step's keys and values [T][kv_heads][head_dim] (views with
    contiguous heads) to the slots (int64 [T]; negative: skipped)."""
    _native.cache_write(cache.k, cache.v, k, v, slots, stream)


def tree_attention(q, cache: KVCache, page_table, context_lens, query_start, tree_mask, max_new: int, scale=None,
                   out=None, workspace=None, stream=None):
    """Attention of a step's tokens q [T][heads][head_dim] over the cache,
    which already holds their keys and values; max_new: the most new tokens of
    a request; scale: 1 / sqrt(head_dim) by default.  Returns [T][heads]
    [head_dim]: 0 in rows of no request (a padded plan's), and NaN in all rows of
    a request that brings more than max_new tokens, as a prompt chunk of more than
    64 does, or more than its row of the table holds.  A given out keeps what it
    has in rows of no request and in those that max_new or the table leave out.
    workspace: a uint8 tensor of
    sbvr_tree_attention_workspace_bytes, by default a new one."""
    return _native.tree_attention(q, cache.k, cache.v, page_table, context_lens, query_start, tree_mask, max_new, scale,
                                  out, workspace, stream)


def residual_norm(x, y=None, post_weight=None, gate=None, scale: float = 1.0, pre_weight=None, eps: float = 1e-5,
                  x_out=None, h_out=None, stream=None):
    """x' = x + scale * gate * rms(y) * post_weight and h = rms(x') *
    pre_weight for tokens x [T][H] (fp16, bf16 or fp32 stream), y [T][H] and
    gate [T][H] or [H] (fp16 or bf16); returns (x', h).  Without pre_weight h
    is None; without y x' is x itself.  x_out may be x."""
    return _native.residual_norm(x, y, post_weight, gate, scale, pre_weight, eps, x_out, h_out, stream)


def adjust_logits(logits, history=None, history_start=None, prompt_lens=None, repetition=None, frequency=None,
                  presence=None, temperature=None, bias_tokens=None, bias_values=None, bias_start=None, grammar=None,
                  grammar_rows=None, token_request=None, query_start=None, tree_mask=None, draft_tokens=None,
                  n_requests=None, out=None, out_dtype=None, stream=None):
    """The logits [T][V] (fp16, bf16 or fp32) with the penalties, biases,
    temperatures and grammar masks of their requests applied (every part
    optional); out may be logits.  One grammar for all rows is a row of it and
    grammar_rows of zeros (its rows must not overlap).  The number of requests R comes from the
    parameters per request or the starts, or n_requests; without token_request
    row t is request t."""
    return _native.adjust_logits(logits, history, history_start, prompt_lens, repetition, frequency, presence,
                                 temperature, bias_tokens, bias_values, bias_start, grammar, grammar_rows, token_request,
                                 query_start, tree_mask, draft_tokens, n_requests, out, out_dtype, stream)
