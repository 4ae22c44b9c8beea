"""Sequence operators of libna.so (``include/na_seq.h``): causal window attention with first
tokens that stay visible, its gradient, and the paged cache that serves it.

Token i attends to token j when ``j <= i`` and (``i - j < kernel_size`` or ``j < sinks``).
Query heads share key/value heads in groups: head h reads key/value head
``h // (heads // kv_heads)``.

Training and prompts, on ``[batch, heads, tokens, head_dim]`` tensors of any batch, head and
token strides (the last axis contiguous):

    out, lse = sink_forward(q, k, v, kernel_size, sinks)
    dq, dk, dv = sink_backward(q, k, v, out, lse, dout, kernel_size, sinks)
    out = sink_attention(q, k, v, kernel_size, sinks)          # under torch.autograd

Serving, one step of a batch of requests over a paged cache:

    cu, slots, positions, head = cache_tables(context_lens, new_lens, page_table, free_pages,
                                              page_size, tokens)
    cache_write(k, v, slots, k_pages, v_pages)
    out, lse = cache_attention(q, k_pages, v_pages, page_table, context_lens, cu)

or the three at once, ``cache_step``; ``serving.py`` has more for long contexts.  Nothing here
synchronises; all work is on the current stream of the tensors' device.
"""
import ctypes
import functools
import math
from operator import index

import torch

from . import DTYPES, _check, _stream, load_library

__all__ = ["sink_forward", "sink_backward", "sink_attention", "cache_tables", "cache_write",
           "cache_attention", "cache_step"]

_vp = ctypes.c_void_p
_i64 = ctypes.c_int64
_WHOLE = (1 << 31) - 1  # kernel_size of attention over the whole context


class _Strides(ctypes.Structure):
    _fields_ = [("batch", _i64), ("head", _i64), ("token", _i64)]


class _SinkProblem(ctypes.Structure):
    _fields_ = ([(n, _i64) for n in ("batch", "heads", "kv_heads", "tokens", "head_dim",
                                     "kernel_size", "sinks")]
                + [(n, _Strides) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")]
                + [("dtype", ctypes.c_int32), ("scale", ctypes.c_float)])


class _CacheProblem(ctypes.Structure):
    _fields_ = ([(n, _i64) for n in ("requests", "tokens", "heads", "kv_heads", "head_dim", "pages",
                                     "page_size", "max_pages", "kernel_size", "sinks", "max_new",
                                     "max_context")]
                + [(n, _Strides) for n in ("q", "k", "v", "out")]
                + [("dtype", ctypes.c_int32), ("scale", ctypes.c_float)])


class _SharedProblem(ctypes.Structure):
    _fields_ = [("cache", _CacheProblem), ("groups", _i64), ("max_shared", _i64),
                ("max_own", _i64)]


class _WeightsProblem(ctypes.Structure):
    _fields_ = [("cache", _CacheProblem), ("capacity", _i64)]


class _EvictProblem(ctypes.Structure):
    _fields_ = ([(n, _i64) for n in ("requests", "kv_heads", "head_dim", "pages", "page_size",
                                     "max_pages", "num_free", "capacity", "budget", "recent")]
                + [("dtype", ctypes.c_int32)])


# argument types of the entry points, without the workspace sizes (ctypes; the problem by pointer)
_SIGNATURES = {
    "na_sink_forward": [ctypes.POINTER(_SinkProblem)] + [_vp] * 7,
    "na_sink_backward": [ctypes.POINTER(_SinkProblem)] + [_vp] * 11 + [ctypes.c_size_t, _vp],
    "na_cache_tables": [_i64] * 5 + [_vp] * 10,
    "na_cache_write": [ctypes.POINTER(_CacheProblem)] + [_vp] * 6,
    "na_cache_attention": [ctypes.POINTER(_CacheProblem)] + [_vp] * 9 + [ctypes.c_size_t, _vp],
    "na_cache_shared_attention": ([ctypes.POINTER(_SharedProblem)] + [_vp] * 11
                                  + [ctypes.c_size_t, _vp]),
    "na_cache_weights": [ctypes.POINTER(_WeightsProblem)] + [_vp] * 9 + [ctypes.c_size_t, _vp],
    "na_cache_evict": [ctypes.POINTER(_EvictProblem)] + [_vp] * 13 + [ctypes.c_size_t, _vp],
}
_WORKSPACES = {
    "na_sink_backward_workspace": _SinkProblem,
    "na_cache_attention_workspace": _CacheProblem,
    "na_cache_shared_attention_workspace": _SharedProblem,
    "na_cache_weights_workspace": _WeightsProblem,
    "na_cache_evict_workspace": _EvictProblem,
}

_bound = None
_entry = {}  # entry points by name: the ctypes function, and how to call it fast (or None)


def _library():
    """libna.so with the argument types of na_seq.h."""
    global _bound, _entry
    lib = load_library()
    if _bound is not lib:
        for name, types in _SIGNATURES.items():
            getattr(lib, name).argtypes = types
        for name, problem in _WORKSPACES.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = [ctypes.POINTER(problem)], ctypes.c_size_t
        try:
            from ._na_fast import call
        except ImportError:
            call = None
        entry = {}
        for name in _SIGNATURES:
            fn = getattr(lib, name)
            if call is None:
                # the problem goes by address in the fast form; ctypes takes it as a pointer
                cast = fn.argtypes[0]
                entry[name] = fn if name == "na_cache_tables" else (
                    lambda p, *args, fn=fn, cast=cast: fn(ctypes.cast(p, cast), *args))
            else:
                entry[name] = functools.partial(call, ctypes.cast(fn, ctypes.c_void_p).value)
        # (another thread may come here at any time: it sees the entries complete, and _bound
        # only after them; two threads that both come first make the same)
        _entry = entry
        _bound = lib
    return lib


# the current device without the checks of torch.cuda.current_device (where torch has it)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(name, device, *args):
    """The entry point with args.. and the current stream of device, that device current."""
    if _device() == device.index:
        status = _entry[name](*args, _stream(device))
    else:
        with torch.cuda.device(device):
            status = _entry[name](*args, _stream(device))
    if status:
        _check(status)


# Checks run once per combination of shapes, strides, types and devices (the functions below
# that are cached take nothing else); addresses are checked by the library, on every call.

def _metas_plain(*tensors):
    """What the checks of each tensor depend on (None: None)."""
    return tuple(None if t is None else (t.shape, t.stride(), t.dtype, t.device) for t in tensors)


try:
    from ._na_fast import metas as _metas
except ImportError:  # (also a build of it without this function)
    _metas = _metas_plain


def _contiguous(shape, stride):
    want = 1
    for n, s in zip(reversed(shape), reversed(stride)):
        if n != 1 and s != want:
            return 0 in shape
        want *= n
    return True


def _rows(*metas):
    """Data tensors: of one supported type, with a contiguous last axis, on one GPU."""
    dtype, device = metas[0][2:]
    if dtype not in DTYPES:
        raise TypeError(f"unsupported dtype {dtype}")
    if any(m[2] != dtype for m in metas):
        raise TypeError("data tensors must share a dtype")
    for m in metas:
        if 0 not in m[0] and m[1][-1] != 1:
            raise ValueError("the last axis must be contiguous")
    for m in metas:
        if m[3].type != "cuda":
            raise ValueError("tensors must live on a GPU")
        if m[3] != device:
            raise ValueError("tensors must share a device")


def _ints(device, dtype, **metas):
    """Integer arrays: contiguous, on the device, of the given type."""
    for name, m in metas.items():
        if m[2] != dtype:
            raise TypeError(f"{name} must be {dtype}")
        if m[3] != device:
            raise ValueError(f"{name} must live on {device}")
        if not _contiguous(m[0], m[1]):
            raise ValueError(f"{name} must be contiguous")


def _check_lse(lse, q):
    if lse is None:
        return
    if lse[2] != torch.float32 or lse[0] != q[0][:-1] or not _contiguous(lse[0], lse[1]):
        raise ValueError("lse must be a contiguous fp32 tensor of shape q.shape[:-1]")
    if lse[3] != q[3]:
        raise ValueError("tensors must share a device")


def _window(kernel_size, sinks, scale):
    """Plain numbers (the plans are looked up by value, never by a tensor's identity)."""
    return (None if kernel_size is None else index(kernel_size), index(sinks),
            None if scale is None else float(scale))


def _bounds(max_new, max_context):
    """The caller's bounds, the second rounded up by at most a tile of 32 keys or 3 %: one that
    grows by a token a step needs a new plan every 32 steps, not every step."""
    if max_context is not None:
        max_context = index(max_context)
        if max_context > 0:
            step = max(5, max_context.bit_length() - 6)
            max_context = -(-max_context >> step) << step
    return None if max_new is None else index(max_new), max_context


def _count(value, name, least):
    if value < least:
        raise ValueError(f"{name} must be at least {least}")
    return min(value, _WHOLE)


def _layout(m):
    """Shape and strides of an output of a tensor's shape and axis order (plain tuples, which
    torch reads faster than its own sizes)."""
    t = torch.empty_like(torch.empty_strided(m[0], m[1], dtype=m[2], device="meta"))
    if t.stride(-1) != 1 and t.numel():
        t = torch.empty(t.shape, device="meta")
    return tuple(t.shape), t.stride()


def _filled(m, ref):
    """The meta of an output: what the caller gave, or what is made for it."""
    return (*_layout(ref), *ref[2:]) if m is None else m


def _lse_shape(q):
    return tuple(q[0][:-1])


# ---------------------------------------------------------------- contiguous sequences

@functools.lru_cache(maxsize=256)
def _sink_plan(kernel_size, sinks, scale, metas):
    """The problem (kept alive by the cache's entry), its address, the layouts of out or of dq,
    dk and dv where the call makes them, and the logsumexp's shape or the backward's workspace.
    metas: of lengths, lse, q, k, v, out[, dout, dq, dk, dv]."""
    lengths, lse, q, k, v, *more = metas
    if len(q[0]) != 4 or len(k[0]) != 4 or k[0] != v[0]:
        raise ValueError("expected q [batch, heads, tokens, head_dim] and k, v of one shape")
    (B, H, N, D), kv_heads = q[0], k[0][1]
    if k[0][0] != B or k[0][2:] != q[0][2:]:
        raise ValueError("q, k and v must share batch, tokens and head_dim")
    if H != kv_heads and (H == 0 or kv_heads == 0 or H % kv_heads):
        raise ValueError("the heads of q must be a multiple of those of k and v")
    _rows(q, k, v, *(m for m in more if m is not None))
    like = (q, q, q, k, v)
    more = [_filled(m, ref) for m, ref in zip(more, like)]
    for m, ref in zip(more, like):
        if m[0] != ref[0]:
            raise ValueError("out, dout and the gradients must have the shapes of q, k and v")
    _check_lse(lse, q)
    if lengths is not None:
        _ints(q[3], torch.int32, lengths=lengths)
        if lengths[0] != (B,):
            raise ValueError("lengths needs one entry per sequence")
    p = _SinkProblem(B, H, kv_heads, N, D, _count(kernel_size, "kernel_size", 1),
                     _count(sinks, "sinks", 0))
    for name, m in zip(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), (q, k, v, *more)):
        setattr(p, name, _Strides(*m[1][:3]))
    p.dtype, p.scale = DTYPES[q[2]], 1.0 / math.sqrt(D) if scale is None else float(scale)
    if len(more) == 1:
        return p, ctypes.addressof(p), _layout(q), _lse_shape(q)
    return (p, ctypes.addressof(p), tuple(_layout(m) for m in (q, k, v)),
            _library().na_sink_backward_workspace(p))


def sink_forward(q, k, v, kernel_size, sinks=0, scale=None, lengths=None, out=None, lse=None):
    """Window attention with visible first tokens.  q [batch, heads, tokens, head_dim], k and v
    [batch, kv_heads, tokens, head_dim]; lengths (int32, on the GPU): valid tokens of each
    sequence of a padded batch.  Returns (out, logsumexp); rows behind a length get 0 and
    -inf."""
    _library()
    p, at, layout, rows = _sink_plan(*_window(kernel_size, sinks, scale),
                                     _metas(lengths, lse, q, k, v, out))
    out = q.new_empty_strided(*layout) if out is None else out
    lse = q.new_empty(rows, dtype=torch.float32) if lse is None else lse
    _call("na_sink_forward", q.device, at, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          0 if lengths is None else lengths.data_ptr(), out.data_ptr(), lse.data_ptr())
    return out, lse


def sink_backward(q, k, v, out, lse, dout, kernel_size, sinks=0, scale=None, lengths=None,
                  dq=None, dk=None, dv=None):
    """Gradients of sink_forward's out with respect to q, k and v, from the out and lse that it
    returned.  Returns (dq, dk, dv), 0 behind a length; the same inputs give the same bits."""
    _library()
    p, at, layouts, need = _sink_plan(*_window(kernel_size, sinks, scale),
                                      _metas(lengths, lse, q, k, v, out, dout, dq, dk, dv))
    dq = q.new_empty_strided(*layouts[0]) if dq is None else dq
    dk = q.new_empty_strided(*layouts[1]) if dk is None else dk
    dv = q.new_empty_strided(*layouts[2]) if dv is None else dv
    # (the allocator hands it out stream by stream, and to a captured graph from its own pool)
    work = torch.empty(need, dtype=torch.uint8, device=q.device)
    _call("na_sink_backward", q.device, at, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          0 if lengths is None else lengths.data_ptr(), out.data_ptr(), lse.data_ptr(),
          dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), work.data_ptr(), need)
    return dq, dk, dv


def _readable(t):
    """t, or a contiguous copy where its strides are none that the kernels read."""
    if t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and all(
            s * t.element_size() % 16 == 0 for s in t.stride()[:-1]):
        return t
    return t.contiguous()


def _gradients(ctx, dout):
    q, k, v, out, lse, lengths = ctx.saved_tensors
    return sink_backward(q, k, v, out, lse, _readable(dout), *ctx.cfg, lengths) + (None,) * 4


# (with create_graph: a second derivative raises; the wrapper costs 10 us that others need not pay)
_gradients_once = torch.autograd.function.once_differentiable(_gradients)


class _SinkFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, kernel_size, sinks, scale, lengths):
        out, lse = sink_forward(q, k, v, kernel_size, sinks, scale, lengths)
        ctx.save_for_backward(q, k, v, out, lse, lengths)
        ctx.cfg = (kernel_size, sinks, scale)
        return out

    @staticmethod
    def backward(ctx, dout):
        return (_gradients_once if torch.is_grad_enabled() else _gradients)(ctx, dout)


def sink_attention(q, k, v, kernel_size, sinks=0, scale=None, lengths=None):
    """Autograd-aware window attention with visible first tokens (see sink_forward).  Capture
    its forward and backward into one graph with no eager autograd graph of the same leaves
    alive: torch runs a leaf's accumulation on the stream of the oldest such graph, which a
    capture of another stream cannot join."""
    return _SinkFunction.apply(q, k, v, kernel_size, sinks, scale, lengths)


# ---------------------------------------------------------------- the paged cache

@functools.lru_cache(maxsize=256)
def _tables_plan(tokens, page_size, metas):
    """Arguments of na_cache_tables up to the arrays.  metas: of context_lens, new_lens,
    page_table, free_pages, head, cu_new, slots, positions and new_head."""
    context, new, table, free, head, *outs = metas
    if len(context[0]) != 1 or new[0] != context[0]:
        raise ValueError("context_lens and new_lens need one entry per request")
    if len(table[0]) != 2 or table[0][0] != context[0][0]:
        raise ValueError("page_table must be [requests, max_pages]")
    if len(free[0]) != 1:
        raise ValueError("free_pages must be one list")
    if context[3].type != "cuda":
        raise ValueError("tensors must live on a GPU")
    requests, device = context[0][0], context[3]
    _ints(device, torch.int32, context_lens=context, new_lens=new, page_table=table,
          free_pages=free)
    if head is not None:
        _ints(device, torch.int32, head=head)
        if head[0].numel() != 1:
            raise ValueError("head needs one entry")
    for name, m, n, dtype in zip(("cu_new", "slots", "positions", "new_head"), outs,
                                 (requests + 1, tokens, tokens, 1),
                                 (torch.int32, torch.int64, torch.int32, torch.int32)):
        if m is not None:
            _ints(device, dtype, **{name: m})
            if m[0] != (n,):
                raise ValueError(f"{name} needs {n} entries")
    return requests, _count(tokens, "tokens", 0), page_size, table[0][1], free[0][0]


def cache_tables(context_lens, new_lens, page_table, free_pages, page_size, tokens, head=None,
                 cu_new=None, slots=None, positions=None, new_head=None):
    """Tables of a step: request r has context_lens[r] tokens cached and gets new_lens[r] more
    (int32, on the GPU).  Pages that the new tokens begin are taken from free_pages from index
    head (int32 [1] on the GPU; None: 0) on and entered into page_table [requests, max_pages].
    `tokens` is the room for new tokens, at least their number.
    Returns (cu_new [requests + 1] int32, slots [tokens] int64, positions [tokens] int32,
    new_head [1] int32); slots and positions behind the last token are -1, and so are the slots
    of tokens whose page the pool (new_head > len(free_pages)) or the table has no room for."""
    _library()
    sizes = _tables_plan(index(tokens), index(page_size),
                         _metas(context_lens, new_lens, page_table, free_pages, head, cu_new,
                                slots, positions, new_head))
    # (like context_lens: int32)
    if cu_new is None:
        cu_new = context_lens.new_empty(sizes[0] + 1)
    if slots is None:
        slots = context_lens.new_empty(sizes[1], dtype=torch.int64)
    if positions is None:
        positions = context_lens.new_empty(sizes[1])
    if new_head is None:
        new_head = context_lens.new_empty(1)
    _call("na_cache_tables", context_lens.device, *sizes, context_lens.data_ptr(), new_lens.data_ptr(),
          free_pages.data_ptr(), 0 if head is None else head.data_ptr(), page_table.data_ptr(),
          cu_new.data_ptr(), slots.data_ptr(), positions.data_ptr(), new_head.data_ptr())
    return cu_new, slots, positions, new_head


def _check_pages(k_pages, v_pages):
    if len(k_pages[0]) != 4 or k_pages[0] != v_pages[0]:
        raise ValueError("pages must be [pages, kv_heads, page_size, head_dim], k and v alike")
    if not (_contiguous(*k_pages[:2]) and _contiguous(*v_pages[:2])):
        raise ValueError("pages must be contiguous")


def _token_strides(m):
    return _Strides(0, m[1][1], m[1][0])


@functools.lru_cache(maxsize=256)
def _write_plan(metas):
    """The problem of na_cache_write (kept alive by the cache's entry) and its address.  metas:
    of k, v, slots, k_pages and v_pages."""
    k, v, slots, k_pages, v_pages = metas
    if len(k[0]) != 3 or k[0] != v[0]:
        raise ValueError("expected k and v [tokens, kv_heads, head_dim]")
    _check_pages(k_pages, v_pages)
    _rows(k, v, k_pages, v_pages)
    if k[0][1:] != k_pages[0][1::2]:
        raise ValueError("k, v and the pages must share kv_heads and head_dim")
    _ints(k[3], torch.int64, slots=slots)
    if slots[0] != k[0][:1]:
        raise ValueError("slots needs one entry per token")
    p = _CacheProblem(0, k[0][0], 0, k[0][1], k[0][2], k_pages[0][0], k_pages[0][2], 0, 1, 0, 0, 0)
    p.k, p.v = _token_strides(k), _token_strides(v)
    p.dtype, p.scale = DTYPES[k[2]], 1.0
    return p, ctypes.addressof(p)


def cache_write(k, v, slots, k_pages, v_pages):
    """Writes row t of k and v [tokens, kv_heads, head_dim] into the pages [pages, kv_heads,
    page_size, head_dim] at slots[t] (page * page_size + offset, int64); slots outside the
    pages (-1) are skipped.  The slots of one call must differ."""
    _library()
    p, at = _write_plan(_metas(k, v, slots, k_pages, v_pages))
    _call("na_cache_write", k.device, at, k.data_ptr(), v.data_ptr(), slots.data_ptr(),
          k_pages.data_ptr(), v_pages.data_ptr())


@functools.lru_cache(maxsize=256)
def _attention_plan(kernel_size, sinks, scale, max_new, max_context, metas):
    """The problem of na_cache_attention (kept alive by the cache's entry), its address, its
    workspace's size, and the layout of out and the logsumexp's shape where the call makes them.
    metas: of q, k_pages, v_pages, page_table, context_lens, cu_new, out and lse."""
    p = _attention_problem(kernel_size, sinks, scale, max_new, max_context, metas)
    q = metas[0]
    return (p, ctypes.addressof(p), _library().na_cache_attention_workspace(p), _layout(q),
            _lse_shape(q))


def _attention_problem(kernel_size, sinks, scale, max_new, max_context, metas):
    """The checks of new tokens against the cache, and their problem."""
    q, k_pages, v_pages, table, context, cu_new, out, lse = metas
    if len(q[0]) != 3:
        raise ValueError("expected q [tokens, heads, head_dim]")
    _check_pages(k_pages, v_pages)
    (T, H, D), (P, kv_heads, page_size, _) = q[0], k_pages[0]
    if D != k_pages[0][3]:
        raise ValueError("q and the pages must share head_dim")
    if H != kv_heads and (H == 0 or kv_heads == 0 or H % kv_heads):
        raise ValueError("the heads of q must be a multiple of those of the pages")
    if len(context[0]) != 1 or len(table[0]) != 2 or table[0][0] != context[0][0]:
        raise ValueError("expected context_lens [requests] and page_table [requests, max_pages]")
    if cu_new[0] != (context[0][0] + 1,):
        raise ValueError("cu_new needs one entry more than there are requests")
    if out is not None and out[0] != q[0]:
        raise ValueError("out must have the shape of q")
    _rows(q, k_pages, v_pages, *(() if out is None else (out,)))
    out = _filled(out, q)
    _check_lse(lse, q)
    _ints(q[3], torch.int32, page_table=table, context_lens=context, cu_new=cu_new)
    p = _CacheProblem(
        context[0][0], T, H, kv_heads, D, P, page_size, table[0][1],
        _WHOLE if kernel_size is None else _count(kernel_size, "kernel_size", 1),
        _count(sinks, "sinks", 0), 0 if max_new is None else _count(max_new, "max_new", 0),
        0 if max_context is None else _count(max_context, "max_context", 0))
    p.q, p.out = _token_strides(q), _token_strides(out)
    p.dtype, p.scale = DTYPES[q[2]], 1.0 / math.sqrt(D) if scale is None else float(scale)
    return p


def cache_attention(q, k_pages, v_pages, page_table, context_lens, cu_new, kernel_size=None,
                    sinks=0, scale=None, max_new=None, max_context=None, out=None, lse=None):
    """Attention of new tokens q [tokens, heads, head_dim] over the cache that already holds
    their keys and values: token t of request r is row cu_new[r] + t, at position
    context_lens[r] + t.  kernel_size None: the whole context.  max_new and max_context, bounds
    of the new tokens and of the whole tokens of any request where the caller knows them, only
    choose how the work is split.  Returns (out, logsumexp [tokens, heads] fp32); rows from
    cu_new[requests] on are left as they were.  A page id outside the pages reads as zeros."""
    _library()
    p, at, need, layout, rows = _attention_plan(
        *_window(kernel_size, sinks, scale), *_bounds(max_new, max_context),
        _metas(q, k_pages, v_pages, page_table, context_lens, cu_new, out, lse))
    out = q.new_empty_strided(*layout) if out is None else out
    lse = q.new_empty(rows, dtype=torch.float32) if lse is None else lse
    # (the allocator hands it out stream by stream, and to a captured graph from its own pool)
    work = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _call("na_cache_attention", q.device, at, q.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), page_table.data_ptr(), context_lens.data_ptr(), cu_new.data_ptr(),
          out.data_ptr(), lse.data_ptr(), work.data_ptr() if need else 0, need)
    return out, lse


@functools.lru_cache(maxsize=256)
def _step_plan(kernel_size, sinks, scale, max_new, max_context, metas):
    """The problem of both the write and the attention of a step (kept alive by the cache's
    entry), its address, its workspace's size, the layout of out and the logsumexp's shape, and
    the arguments of na_cache_tables; the checks are those of the three functions.  metas: of
    q, k, v, k_pages, v_pages, page_table, context_lens, then of new_lens, free_pages and head,
    or of the cu_new and slots that the caller has."""
    q, k, v, k_pages, v_pages, page_table, context, *more = metas
    if len(q[0]) != 3 or len(k[0]) != 3 or q[0][0] != k[0][0]:
        raise ValueError("q, k and v need the same new tokens")
    T, device = q[0][0], q[3]
    sizes, requests = None, context[0][0] if len(context[0]) == 1 else 0
    _check_pages(k_pages, v_pages)
    if len(more) == 3:
        new, free, head = more
        sizes = _tables_plan.__wrapped__(T, k_pages[0][2], (context, new, page_table, free, head)
                                         + (None,) * 4)
        ints = lambda n, dtype: (torch.Size((n,)), (1,), dtype, device)  # noqa: E731
        more = ints(requests + 1, torch.int32), ints(T, torch.int64)
    cu_new, slots = more
    _write_plan.__wrapped__((k, v, slots, k_pages, v_pages))
    p, at, need, layout, rows = _attention_plan.__wrapped__(
        kernel_size, sinks, scale, max_new, max_context,
        (q, k_pages, v_pages, page_table, context, cu_new, None, None))
    _rows(q, k)
    p.k, p.v = _token_strides(k), _token_strides(v)
    return p, at, need, layout, rows, sizes


def cache_step(q, k, v, k_pages, v_pages, page_table, context_lens, new_lens, free_pages,
               kernel_size=None, sinks=0, scale=None, head=None, max_new=None, max_context=None,
               tables=None):
    """One serving step of an attention layer: the tables of the new tokens, their keys and
    values into the pages, and their attention.  q [tokens, heads, head_dim], k and v [tokens,
    kv_heads, head_dim] hold the requests' new tokens one after another.  `tables`: what
    cache_tables returned for this step (the layers of a model share it); None builds it.
    Returns (out, logsumexp, new_head); rows of out behind the last new token are not written."""
    _library()
    device = q.device
    if tables is None:
        metas = _metas(q, k, v, k_pages, v_pages, page_table, context_lens, new_lens, free_pages,
                       head)
    else:
        cu_new, slots, _, new_head = tables
        metas = _metas(q, k, v, k_pages, v_pages, page_table, context_lens, cu_new, slots)
    p, at, need, layout, rows, sizes = _step_plan(
        *_window(kernel_size, sinks, scale), *_bounds(max_new, max_context), metas)
    out = q.new_empty_strided(*layout)
    lse = q.new_empty(rows, dtype=torch.float32)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    context, table = context_lens.data_ptr(), page_table.data_ptr()
    kp, vp = k_pages.data_ptr(), v_pages.data_ptr()
    if tables is None:
        # slots, positions and cu_new live in one buffer (only the new head is handed out)
        tokens = sizes[1]
        ints = context_lens.new_empty(3 * tokens + sizes[0] + 1)
        new_head = context_lens.new_empty(1)
        slots = ints.data_ptr()
        positions, cu_new = slots + 8 * tokens, slots + 12 * tokens
        _call("na_cache_tables", device, *sizes, context, new_lens.data_ptr(),
              free_pages.data_ptr(), 0 if head is None else head.data_ptr(), table, cu_new, slots,
              positions, new_head.data_ptr())
    else:
        cu_new, slots = cu_new.data_ptr(), slots.data_ptr()
    _call("na_cache_write", device, at, k.data_ptr(), v.data_ptr(), slots, kp, vp)
    _call("na_cache_attention", device, at, q.data_ptr(), kp, vp, table, context, cu_new,
          out.data_ptr(), lse.data_ptr(), work.data_ptr() if need else 0, need)
    return out, lse, new_head
