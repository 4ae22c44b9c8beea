"""Cache operators for long contexts (``include/na_seq.h``), beside the paged cache of
``sequence.py``: attention of requests that share their first tokens, the attention weight that
cached keys gather, and the eviction of those that gathered least.

A serving loop over a cache whose requests share a system prompt:

    cu, slots, positions, head = cache_tables(context_lens, new_lens, page_table, free_pages,
                                              page_size, tokens, head)
    cache_write(k, v, slots, k_pages, v_pages)
    out, lse = cache_shared_attention(q, k_pages, v_pages, page_table, context_lens, cu,
                                      cu_groups, shared_lens)
    cache_weights(q, lse, k_pages, page_table, context_lens, cu, weights, first=prompt_lens)
    context_lens += new_lens
    # now and then
    context_lens, weights, kept, head = cache_evict(weights, k_pages, v_pages, page_table,
                                                    context_lens, free_pages, head, budget,
                                                    recent, first=prompt_lens)

Pass max_new (and max_shared and max_own, max_context) where they are known: without them a
batch of single tokens takes the forms for chunks, 1.5 to 1.7 times as long.  Nothing here
synchronises; all work is on the current stream of the tensors' device.
"""
import ctypes
import functools
from operator import index

import torch

from . import DTYPES, _check
from .sequence import (_attention_problem, _bounds, _call, _check_pages, _contiguous, _count,
                       _EvictProblem, _ints, _layout, _library, _lse_shape, _metas, _rows,
                       _SharedProblem, _WeightsProblem, _window)

__all__ = ["cache_shared_attention", "cache_weights", "cache_evict"]

_ERR_NULL = 1  # NA_ERR_NULL


@functools.lru_cache(maxsize=256)
def _shared_plan(kernel_size, sinks, scale, max_new, max_shared, max_own, metas):
    """The problem of na_cache_shared_attention (kept alive by the cache's entry), its address, its
    workspace's size, and the layout of out and the logsumexp's shape where the call makes them.
    metas: of q, k_pages, v_pages, page_table, context_lens, cu_new, out, lse, cu_groups and
    shared_lens."""
    *cache, cu_groups, shared = metas
    q = cache[0]
    problem = _attention_problem(kernel_size, sinks, scale, max_new, None, tuple(cache))
    _ints(q[3], torch.int32, cu_groups=cu_groups, shared_lens=shared)
    if len(shared[0]) != 1 or cu_groups[0] != (shared[0][0] + 1,):
        raise ValueError("expected shared_lens [groups] and cu_groups [groups + 1]")
    s = _SharedProblem(problem, shared[0][0],
                       0 if max_shared is None else _count(max_shared, "max_shared", 0),
                       0 if max_own is None else _count(max_own, "max_own", 0))
    return (s, ctypes.addressof(s), _library().na_cache_shared_attention_workspace(s), _layout(q),
            _lse_shape(q))


def cache_shared_attention(q, k_pages, v_pages, page_table, context_lens, cu_new, cu_groups,
                           shared_lens, kernel_size=None, sinks=0, scale=None, max_new=None,
                           max_shared=None, max_own=None, out=None, lse=None):
    """cache_attention of a batch in which groups of requests share their first tokens: the shared
    keys and values are read once for all rows of a group.  Requests cu_groups[g] ..
    cu_groups[g + 1] - 1 (int32, on the GPU, not decreasing) share their first shared_lens[g]
    tokens, which are read on the pages of the first of them; the others are read on each
    request's own pages.  Requests outside of all groups share nothing.  max_new, max_shared and
    max_own, bounds of the new tokens of a request, of the shared ones of a group and of a
    request's tokens behind those (the new ones among them), only choose how the work is split.
    It pays where many rows meet the shared keys: single or a few new tokens of many requests.  For
    chunks of prompts cache_attention, over tables that list the shared pages, takes as long.  A row
    that sees a key with a score of NaN or +inf gets NaN.
    Returns (out, logsumexp [tokens, heads] fp32); rows from cu_new[requests] on are left as they
    were."""
    _library()
    p, at, need, layout, rows = _shared_plan(
        *_window(kernel_size, sinks, scale), *_bounds(max_new, max_shared),
        _bounds(None, max_own)[1],
        _metas(q, k_pages, v_pages, page_table, context_lens, cu_new, out, lse, cu_groups,
               shared_lens))
    out = q.new_empty_strided(*layout) if out is None else out
    lse = q.new_empty(rows, dtype=torch.float32) if lse is None else lse
    # (the allocator hands it out stream by stream, and to a captured graph from its own pool)
    work = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _call("na_cache_shared_attention", q.device, at, q.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), page_table.data_ptr(), context_lens.data_ptr(), cu_new.data_ptr(),
          cu_groups.data_ptr(), shared_lens.data_ptr(), out.data_ptr(), lse.data_ptr(),
          work.data_ptr() if need else 0, need)
    return out, lse


def _check_weights(name, m, requests, kv_heads, device):
    if m[2] != torch.float32:
        raise TypeError(f"{name} must be torch.float32")
    if len(m[0]) != 3 or m[0][:2] != (requests, kv_heads):
        raise ValueError(f"{name} must be [requests, kv_heads, capacity]")
    if m[3] != device:
        raise ValueError(f"{name} must live on {device}")
    if not _contiguous(m[0], m[1]):
        raise ValueError(f"{name} must be contiguous")


def _check_first(first, requests, device):
    if first is not None:
        _ints(device, torch.int32, first=first)
        if first[0] != (requests,):
            raise ValueError("first needs one entry per request")


@functools.lru_cache(maxsize=256)
def _weights_plan(kernel_size, sinks, scale, max_new, max_context, metas):
    """The problem of na_cache_weights (kept alive by the cache's entry), its address and its
    workspace's size.  metas: of q, lse, k_pages, page_table, context_lens, cu_new, weights and
    first."""
    q, lse, k_pages, table, context, cu_new, weights, first = metas
    if lse is None:
        raise ValueError("lse is needed")
    problem = _attention_problem(kernel_size, sinks, scale, max_new, max_context,
                                 (q, k_pages, k_pages, table, context, cu_new, None, lse))
    _check_weights("weights", weights, context[0][0], k_pages[0][1], q[3])
    _check_first(first, context[0][0], q[3])
    p = _WeightsProblem(problem, weights[0][2])
    return p, ctypes.addressof(p), _library().na_cache_weights_workspace(p)


def cache_weights(q, lse, k_pages, page_table, context_lens, cu_new, weights, kernel_size=None,
                  sinks=0, scale=None, first=None, max_new=None, max_context=None):
    """Adds up the attention weights that the keys of the cache get from new tokens q [tokens,
    heads, head_dim], whose keys the cache holds already: weights[r, c, j] (fp32 [requests,
    kv_heads, capacity], updated) gathers exp(scale q . k - lse) over the new tokens of request r
    that see position j and the query heads of key/value head c.  lse [tokens, heads]: what
    cache_attention or cache_shared_attention returned for them, with the same kernel_size,
    sinks and scale.  Entries before first[r] (int32 [requests]; None: 0) are left as they
    were, though their keys are read.  All keys are read on each request's own pages.  Start a
    request's entries at 0."""
    _library()
    p, at, need = _weights_plan(*_window(kernel_size, sinks, scale), *_bounds(max_new, max_context),
                                _metas(q, lse, k_pages, page_table, context_lens, cu_new, weights,
                                       first))
    work = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _call("na_cache_weights", q.device, at, q.data_ptr(), lse.data_ptr(), k_pages.data_ptr(),
          page_table.data_ptr(), context_lens.data_ptr(), cu_new.data_ptr(),
          0 if first is None else first.data_ptr(), weights.data_ptr(),
          work.data_ptr() if need else 0, need)


@functools.lru_cache(maxsize=256)
def _evict_plan(budget, recent, metas):
    """The problem of na_cache_evict (kept alive by the cache's entry), its address and its
    workspace's size.  metas: of weights, k_pages, v_pages, page_table, context_lens, free_pages,
    head and first."""
    weights, k_pages, v_pages, table, context, free, head, first = metas
    _check_pages(k_pages, v_pages)
    _rows(k_pages, v_pages)
    device = k_pages[3]
    P, kv_heads, page_size, D = k_pages[0]
    if len(context[0]) != 1 or len(table[0]) != 2 or table[0][0] != context[0][0]:
        raise ValueError("expected context_lens [requests] and page_table [requests, max_pages]")
    if len(free[0]) != 1:
        raise ValueError("free_pages must be one list")
    _ints(device, torch.int32, page_table=table, context_lens=context, free_pages=free, head=head)
    if head[0].numel() != 1:
        raise ValueError("head needs one entry")
    _check_weights("weights", weights, context[0][0], kv_heads, device)
    _check_first(first, context[0][0], device)
    p = _EvictProblem(context[0][0], kv_heads, D, P, page_size, table[0][1], free[0][0],
                      weights[0][2], _count(budget, "budget", 1), _count(recent, "recent", 0),
                      DTYPES[k_pages[2]])
    # (without pointers: what the library refuses of the problem itself it refuses before those, and
    # here before the call's outputs, which have its sizes, are allocated)
    status = _library().na_cache_evict(p, *[None] * 13, 0, None)
    if status != _ERR_NULL:
        _check(status)
    return p, ctypes.addressof(p), _library().na_cache_evict_workspace(p)


def cache_evict(weights, k_pages, v_pages, page_table, context_lens, free_pages, head, budget,
                recent=0, first=None):
    """Cuts the requests of a cache back to `budget` tokens a key/value head: of a longer one every
    head keeps the first first[r] tokens (int32 [requests]; None: 0), the last `recent` ones and
    those of the others with the largest weight (of equal ones the earlier), `budget` in all.
    The first stay where they are, the last ones end up in front of position `budget` in order,
    and of the others those that lie behind their part of the positions fill the places of those
    that go, in order; keys and values move with them, on the request's own pages.  Pages that
    are no longer needed return to free_pages below index head (int32 [1]).  Requests may share
    pages that hold nothing but tokens before min(first[r], budget); a page with any token behind
    them belongs to one request.
    Returns (context_lens, weights, kept, head): the lengths after it, the weights that moved along
    (0 behind the tokens), for every position the one that its token had (int32 [requests,
    kv_heads, budget], -1 behind the tokens) and the free list's new head.  page_table is left as
    it is; its entries behind a request's tokens mean nothing any more.  Positions are places in
    the cache from then on: cache_tables counts a request's new tokens on from its shortened
    length, and kernel_size counts places.  Where keys are rotated by their tokens' places in the
    text, keep those beside the cache (kept says where a place's token was), and rotate new
    tokens by them, not by the positions of cache_tables."""
    _library()
    p, at, need = _evict_plan(index(budget), index(recent),
                              _metas(weights, k_pages, v_pages, page_table, context_lens,
                                     free_pages, head, first))
    device = weights.device
    new_context = torch.empty_like(context_lens)
    new_weights = torch.empty_like(weights)
    kept = context_lens.new_empty((p.requests, p.kv_heads, p.budget))
    new_head = context_lens.new_empty(1)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _call("na_cache_evict", device, at, weights.data_ptr(), context_lens.data_ptr(),
          0 if first is None else first.data_ptr(), page_table.data_ptr(), head.data_ptr(),
          free_pages.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), new_context.data_ptr(),
          new_weights.data_ptr(), kept.data_ptr(), new_head.data_ptr(),
          work.data_ptr() if need else 0, need)
    return new_context, new_weights, kept, new_head
