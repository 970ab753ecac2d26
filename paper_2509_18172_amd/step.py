"""The operators between the products of a step, on torch tensors: the plan of
a batch, the paged key/value cache, attention for trees of drafted tokens, the
norms around a block and the adjustment of logits; the rotation of queries and
keys, the selection of a beam search and the pages that its sequences share
(include/sbvr.h says what each computes).  Marshalling only, as the package's other helpers: shapes are
checked (AssertionError), outputs come from torch, and a non-zero status raises
``SBVRError``.  The helpers themselves are native (csrc/step_bind.cpp).

A step in order: ``batch_plan`` (pages, slots, masks), per layer
``residual_norm`` -> products -> ``rotary_write`` (or ``rotary`` and
``cache_write``) -> ``tree_attention`` -> products, and ``adjust_logits`` on the
last product.  With beams, a row of the page table is a beam: ``page_usage``
gives the free pages before the plan, and after the logits ``beam_select``,
``page_fork`` and ``page_copy`` make the next step's rows.  ``stream``: a
torch.cuda.Stream of the tensors' device, by default its current one; the call
is made with that device and stream as the current ones, so outputs and
workspaces belong to the stream as they do under ``torch.cuda.stream(stream)``.

Forward only: results carry no gradient, whatever the inputs say, and what is
written in place (page_table, a cache, x_out, out) is not marked as changed.
(A rotation's gradient is the inverse rotation of the outputs' gradients.)
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
             "sbvr_tree_attention_whole", "sbvr_residual_norm", "sbvr_adjust_logits", "sbvr_rotary", "sbvr_rotary_write",
             "sbvr_beam_select_workspace_bytes", "sbvr_beam_select", "sbvr_page_usage_workspace_bytes", "sbvr_page_usage",
             "sbvr_page_fork", "sbvr_page_compact_workspace_bytes", "sbvr_page_compact", "sbvr_page_copy")


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


def rotary(q, k, positions, frequencies, axes=None, interleaved: bool = False, inverse: bool = False, q_out=None,
           k_out=None, stream=None):
    """Queries and keys [T][heads][head_dim] (fp16, bf16 or fp32, views with
    contiguous heads; either may be None) turned by their positions: int32 [T],
    or [axes][T] (one row expanded among them) with axes (int32 [pairs]) naming
    each pair's.  frequencies: fp32 [pairs], the angle per position; the
    elements behind the pairs are copied.  Pairs are element i and i + pairs, or
    neighbours (interleaved); inverse turns back.  Returns (q, k); q_out may be
    q, k_out k."""
    return _native.rotary(q, k, positions, frequencies, axes, interleaved, inverse, q_out, k_out, stream)


def rotary_write(q, cache: KVCache, k, v, slots, positions, frequencies, axes=None, interleaved: bool = False,
                 inverse: bool = False, q_out=None, stream=None):
    """``rotary`` and ``cache_write`` in one pass: the turned keys and the
    values go to their slots of the cache, the turned queries (None: none) are
    returned."""
    return _native.rotary_write(q, cache.k, cache.v, k, v, slots, positions, frequencies, axes, interleaved, inverse, q_out,
                                stream)


class BeamChoice:
    """What ``beam_select`` returns: device tensors tokens, parents int32 and
    scores fp32 [R][n] of the best continuations; ended fp32 and ended_tokens
    int32 [R][B], a beam's score and token if it ends (-infinity, -1: not)."""
    __slots__ = ("tokens", "parents", "scores", "ended", "ended_tokens")

    def __init__(self, tokens, parents, scores, ended, ended_tokens):
        self.tokens, self.parents, self.scores = tokens, parents, scores
        self.ended, self.ended_tokens = ended, ended_tokens


def beam_select(logits, scores, n=None, end_tokens=None, out=None, workspace=None, stream=None) -> BeamChoice:
    """The n (default: as many as beams) best continuations of each request's
    beams: logits [R * B][V] (fp16, bf16 or fp32), scores fp32 [R][B] the
    beams' log probabilities (-infinity: no such beam), end_tokens int32 [E]:
    tokens that end a beam.  out: a BeamChoice of the same sizes to fill, whose
    scores may be the old ones where n is their number; workspace: a uint8
    tensor of sbvr_beam_select_workspace_bytes, by default a new one."""
    given = None if out is None else [getattr(out, name) for name in BeamChoice.__slots__]
    made = _native.beam_select(logits, scores, n, end_tokens, given, workspace, stream)
    return BeamChoice(*made) if out is None else out


class PageUsage:
    """What ``page_usage`` returns: device tensors int32, refs [n_pages] how
    many rows use a page, free_pages [n_pages] the unused ones and then -1,
    counts [2] free and used pages."""
    __slots__ = ("refs", "free_pages", "counts")

    def __init__(self, refs, free_pages, counts):
        self.refs, self.free_pages, self.counts = refs, free_pages, counts


def page_usage(context_lens, page_table, page_size: int, n_pages: int, out=None, workspace=None, stream=None) -> PageUsage:
    """Which of a cache's n_pages pages the rows (context_lens int32 [R],
    page_table int32 [R][max_pages]) use, and which are free.  out: a PageUsage
    of the same sizes to fill; workspace: a uint8 tensor of
    sbvr_page_usage_workspace_bytes, by default a new one."""
    given = None if out is None else [getattr(out, name) for name in PageUsage.__slots__]
    made = _native.page_usage(context_lens, page_table, page_size, n_pages, given, workspace, stream)
    return PageUsage(*made) if out is None else out


class PageFork:
    """What ``page_fork`` returns: device tensors int32, page_table [N]
    [max_pages] and context_lens [N] of the new rows, src, dst and tokens [N]
    (the copies that ``page_copy`` has to make), used [1] pages needed."""
    __slots__ = ("page_table", "context_lens", "src", "dst", "tokens", "used")

    def __init__(self, page_table, context_lens, src, dst, tokens, used):
        self.page_table, self.context_lens = page_table, context_lens
        self.src, self.dst, self.tokens, self.used = src, dst, tokens, used


def page_fork(context_lens, page_table, parents, page_size: int, free_pages, taken=None, out=None, stream=None) -> PageFork:
    """New rows that continue old ones: parents int32 [groups][rows of a group]
    numbers each new row's parent within its group of the old rows
    (context_lens int32 [R], page_table int32 [R][max_pages], R a multiple of
    the groups); any other number makes an empty row.  Full pages are shared, a
    partly filled one is copied into one of free_pages for all but the first of
    a parent's rows; taken (int32, its first element counts): how many of
    free_pages are gone.  out: a PageFork of the same sizes to fill, of which
    nothing may be an input (a captured step forks from one into another)."""
    given = None if out is None else [getattr(out, name) for name in PageFork.__slots__]
    made = _native.page_fork(context_lens, page_table, parents, page_size, free_pages, taken, given, stream)
    return PageFork(*made) if out is None else out


class PageCompaction:
    """What ``page_compact`` returns: device tensors int32, page_table [R]
    [max_pages], src and dst [n_pages // 2] (the moves that ``page_copy`` has to
    make), counts [2] pages in use and pages moved."""
    __slots__ = ("page_table", "src", "dst", "counts")

    def __init__(self, page_table, src, dst, counts):
        self.page_table, self.src, self.dst, self.counts = page_table, src, dst, counts


def page_compact(context_lens, page_table, page_size: int, n_pages: int, out=None, workspace=None,
                 stream=None) -> PageCompaction:
    """New numbers for the pages in use, so that they are the lowest ones.
    Arguments as ``page_usage``; out: a PageCompaction of the same sizes to
    fill, whose page_table may be the old one; workspace: a uint8 tensor of
    sbvr_page_compact_workspace_bytes, by default a new one."""
    given = None if out is None else [getattr(out, name) for name in PageCompaction.__slots__]
    made = _native.page_compact(context_lens, page_table, page_size, n_pages, given, workspace, stream)
    return PageCompaction(*made) if out is None else out


def page_copy(caches, src, dst, tokens=None, stream=None):
    """Copy the first tokens[i] tokens (int32 [n]; None: all) of page src[i] to
    page dst[i] (int32 [n]; negative: skipped), in each of the caches: one
    KVCache, or a sequence of them, alike but for their memory."""
    caches = [caches] if isinstance(caches, KVCache) else list(caches)
    _native.page_copy([c.k for c in caches], [c.v for c in caches], src, dst, tokens, stream)
