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

or the three at once, ``cache_step``.  Nothing here synchronises; all work is on the current
stream of the tensors' device.
"""
import ctypes
import functools
import math

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


_bound = None


def _library():
    """libna.so with the argument types of na_seq.h."""
    global _bound
    lib = load_library()
    if _bound is not lib:
        sink, cache = ctypes.POINTER(_SinkProblem), ctypes.POINTER(_CacheProblem)
        lib.na_sink_forward.argtypes = [sink] + [_vp] * 7
        lib.na_sink_backward.argtypes = [sink] + [_vp] * 11 + [ctypes.c_size_t, _vp]
        lib.na_sink_backward_workspace.argtypes = [sink]
        lib.na_sink_backward_workspace.restype = ctypes.c_size_t
        lib.na_cache_tables.argtypes = [_i64] * 5 + [_vp] * 10
        lib.na_cache_write.argtypes = [cache] + [_vp] * 6
        lib.na_cache_attention.argtypes = ([cache] + [_vp] * 9 + [ctypes.c_size_t, _vp])
        lib.na_cache_attention_workspace.argtypes = [cache]
        lib.na_cache_attention_workspace.restype = ctypes.c_size_t
        _bound = lib
    return lib


def _call(fn, device, *args):
    """fn(args.., current stream of device), with that device current."""
    if torch.cuda.current_device() == device.index:
        _check(fn(*args, _stream(device)))
    else:
        with torch.cuda.device(device):
            _check(fn(*args, _stream(device)))


def _on_gpu(*tensors):
    for t in tensors:
        if not t.is_cuda:
            raise ValueError("tensors must live on a GPU")
        if t.device != tensors[0].device:
            raise ValueError("tensors must share a device")


def _rows(ref, *others):
    """Data tensors: on one GPU, of one supported type, with a contiguous last axis."""
    if ref.dtype not in DTYPES:
        raise TypeError(f"unsupported dtype {ref.dtype}")
    for t in others:
        if t.dtype != ref.dtype:
            raise TypeError("data tensors must share a dtype")
    for t in (ref,) + others:
        if t.numel() and t.stride(-1) != 1:
            raise ValueError("the last axis must be contiguous")
    _on_gpu(ref, *others)


def _ints(ref, dtype, **tensors):
    """Integer arrays beside ref: contiguous, on its device, of the given type."""
    for name, t in tensors.items():
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}")
        if t.device != ref.device:
            raise ValueError(f"{name} must live on {ref.device}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _count(value, name, least):
    value = int(value)
    if value < least:
        raise ValueError(f"{name} must be at least {least}")
    return min(value, _WHOLE)


def _like(t):
    """An output of t's shape and axis order."""
    out = torch.empty_like(t)
    return out if out.stride(-1) == 1 or not out.numel() else torch.empty(
        t.shape, dtype=t.dtype, device=t.device)


# ---------------------------------------------------------------- contiguous sequences

@functools.lru_cache(maxsize=256)
def _sink_problem(shape, kv_heads, kernel_size, sinks, dtype, scale, strides):
    """strides: of q, k, v, out[, dout, dq, dk, dv], each (batch, head, token, 1).  With the
    backward's workspace size, where its strides are there."""
    p = _SinkProblem(shape[0], shape[1], kv_heads, shape[2], shape[3], kernel_size, sinks)
    for name, s in zip(("q", "k", "v", "out", "dout", "dq", "dk", "dv"), strides):
        setattr(p, name, _Strides(*s[:3]))
    p.dtype, p.scale = DTYPES[dtype], scale
    return p, _library().na_sink_backward_workspace(p) if len(strides) > 4 else 0


def _sink_args(q, k, v, kernel_size, sinks, scale, lengths):
    if q.dim() != 4 or k.dim() != 4 or k.shape != v.shape:
        raise ValueError("expected q [batch, heads, tokens, head_dim] and k, v of one shape")
    if k.shape[0] != q.shape[0] or k.shape[2:] != q.shape[2:]:
        raise ValueError("q, k and v must share batch, tokens and head_dim")
    if q.shape[1] != k.shape[1] and (k.shape[1] == 0 or q.shape[1] % k.shape[1]):
        raise ValueError("the heads of q must be a multiple of those of k and v")
    _rows(q, k, v)
    if lengths is not None:
        _ints(q, torch.int32, lengths=lengths)
        if lengths.shape != q.shape[:1]:
            raise ValueError("lengths needs one entry per sequence")
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    return _count(kernel_size, "kernel_size", 1), _count(sinks, "sinks", 0), float(scale)


def _check_lse(lse, q):
    if lse.dtype != torch.float32 or lse.shape != q.shape[:-1] or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous fp32 tensor of shape q.shape[:-1]")
    _on_gpu(q, lse)


def sink_forward(q, k, v, kernel_size, sinks=0, scale=None, lengths=None, out=None, lse=None):
    """Window attention with visible first tokens.  q [batch, heads, tokens, head_dim], k and v
    [batch, kv_heads, tokens, head_dim]; lengths (int32, on the GPU): valid tokens of each
    sequence of a padded batch.  Returns (out, logsumexp); rows behind a length get 0 and
    -inf."""
    lib = _library()
    kernel_size, sinks, scale = _sink_args(q, k, v, kernel_size, sinks, scale, lengths)
    out = _like(q) if out is None else out
    if lse is None:
        lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    _rows(q, out)
    _check_lse(lse, q)
    p, _ = _sink_problem(q.shape, k.shape[1], kernel_size, sinks, q.dtype, scale,
                         (q.stride(), k.stride(), v.stride(), out.stride()))
    _call(lib.na_sink_forward, q.device, p, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          0 if lengths is None else lengths.data_ptr(), out.data_ptr(), lse.data_ptr())
    return out, lse


def sink_backward(q, k, v, out, lse, dout, kernel_size, sinks=0, scale=None, lengths=None,
                  dq=None, dk=None, dv=None):
    """Gradients of sink_forward's out with respect to q, k and v, from the out and lse that it
    returned.  Returns (dq, dk, dv), 0 behind a length; the same inputs give the same bits."""
    lib = _library()
    kernel_size, sinks, scale = _sink_args(q, k, v, kernel_size, sinks, scale, lengths)
    dq = _like(q) if dq is None else dq
    dk = _like(k) if dk is None else dk
    dv = _like(v) if dv is None else dv
    for t, ref in ((out, q), (dout, q), (dq, q), (dk, k), (dv, k)):
        if t.shape != ref.shape:
            raise ValueError("out, dout and the gradients must have the shapes of q, k and v")
    _rows(q, out, dout, dq, dk, dv)
    _check_lse(lse, q)
    p, need = _sink_problem(q.shape, k.shape[1], kernel_size, sinks, q.dtype, scale,
                            tuple(t.stride() for t in (q, k, v, out, dout, dq, dk, dv)))
    # (the allocator hands it out stream by stream, and to a captured graph from its own pool)
    work = torch.empty(need, dtype=torch.uint8, device=q.device)
    _call(lib.na_sink_backward, q.device, p, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          0 if lengths is None else lengths.data_ptr(), out.data_ptr(), lse.data_ptr(),
          dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), work.data_ptr(), need)
    return dq, dk, dv


def _readable(t):
    """t, or a contiguous copy where its strides are none that the kernels read."""
    if t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and all(
            s * t.element_size() % 16 == 0 for s in t.stride()[:-1]):
        return t
    return t.contiguous()


class _SinkFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, kernel_size, sinks, scale, lengths):
        out, lse = sink_forward(q, k, v, kernel_size, sinks, scale, lengths)
        ctx.save_for_backward(q, k, v, out, lse, lengths)
        ctx.cfg = (kernel_size, sinks, scale)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse, lengths = ctx.saved_tensors
        grads = sink_backward(q, k, v, out, lse, _readable(dout), *ctx.cfg, lengths)
        return grads + (None,) * 4


def sink_attention(q, k, v, kernel_size, sinks=0, scale=None, lengths=None):
    """Autograd-aware window attention with visible first tokens (see sink_forward)."""
    return _SinkFunction.apply(q, k, v, kernel_size, sinks, scale, lengths)


# ---------------------------------------------------------------- the paged cache

@functools.lru_cache(maxsize=256)
def _cache_problem(requests, tokens, heads, kv_heads, head_dim, pages, page_size, max_pages,
                   kernel_size, sinks, max_new, max_context, dtype, scale, strides):
    """strides: of q, k, v, out, each (token, head, 1) or None.  With the workspace's size."""
    p = _CacheProblem(requests, tokens, heads, kv_heads, head_dim, pages, page_size, max_pages,
                      kernel_size, sinks, max_new, max_context)
    for name, s in zip(("q", "k", "v", "out"), strides):
        if s is not None:
            setattr(p, name, _Strides(0, s[1], s[0]))
    p.dtype, p.scale = DTYPES[dtype], scale
    return p, _library().na_cache_attention_workspace(p)


def _check_pages(ref, k_pages, v_pages):
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape:
        raise ValueError("pages must be [pages, kv_heads, page_size, head_dim], k and v alike")
    if not (k_pages.is_contiguous() and v_pages.is_contiguous()):
        raise ValueError("pages must be contiguous")
    _rows(ref, k_pages, v_pages)


def cache_tables(context_lens, new_lens, page_table, free_pages, page_size, tokens, head=None,
                 cu_new=None, slots=None, positions=None, new_head=None):
    """Tables of a step: request r has context_lens[r] tokens cached and gets new_lens[r] more
    (int32, on the GPU).  Pages that the new tokens begin are taken from free_pages from index
    head (int32 [1] on the GPU; None: 0) on and entered into page_table [requests, max_pages].
    `tokens` is the room for new tokens, at least their number.
    Returns (cu_new [requests + 1] int32, slots [tokens] int64, positions [tokens] int32,
    new_head [1] int32); slots and positions behind the last token are -1, and so are the slots
    of tokens whose page the pool (new_head > len(free_pages)) or the table has no room for."""
    lib = _library()
    if context_lens.dim() != 1 or new_lens.shape != context_lens.shape:
        raise ValueError("context_lens and new_lens need one entry per request")
    if page_table.dim() != 2 or page_table.shape[0] != context_lens.shape[0]:
        raise ValueError("page_table must be [requests, max_pages]")
    if free_pages.dim() != 1:
        raise ValueError("free_pages must be one list")
    _on_gpu(context_lens)
    requests, tokens, device = context_lens.shape[0], _count(tokens, "tokens", 0), context_lens.device

    def room(t, n, dtype, name):
        if t is None:
            return torch.empty(n, dtype=dtype, device=device)
        if t.shape != (n,):
            raise ValueError(f"{name} needs {n} entries")
        return t

    cu_new = room(cu_new, requests + 1, torch.int32, "cu_new")
    slots = room(slots, tokens, torch.int64, "slots")
    positions = room(positions, tokens, torch.int32, "positions")
    new_head = room(new_head, 1, torch.int32, "new_head")
    _ints(context_lens, torch.int32, context_lens=context_lens, new_lens=new_lens,
          page_table=page_table, free_pages=free_pages, cu_new=cu_new, positions=positions,
          new_head=new_head)
    _ints(context_lens, torch.int64, slots=slots)
    if head is not None:
        _ints(context_lens, torch.int32, head=head)
        if head.numel() != 1:
            raise ValueError("head needs one entry")
    _call(lib.na_cache_tables, device, requests, tokens, int(page_size), page_table.shape[1],
          free_pages.shape[0], context_lens.data_ptr(), new_lens.data_ptr(),
          free_pages.data_ptr(), 0 if head is None else head.data_ptr(), page_table.data_ptr(),
          cu_new.data_ptr(), slots.data_ptr(), positions.data_ptr(), new_head.data_ptr())
    return cu_new, slots, positions, new_head


def cache_write(k, v, slots, k_pages, v_pages):
    """Writes row t of k and v [tokens, kv_heads, head_dim] into the pages [pages, kv_heads,
    page_size, head_dim] at slots[t] (page * page_size + offset, int64); slots outside the
    pages (-1) are skipped.  The slots of one call must differ."""
    lib = _library()
    if k.dim() != 3 or k.shape != v.shape:
        raise ValueError("expected k and v [tokens, kv_heads, head_dim]")
    _rows(k, v)
    _check_pages(k, k_pages, v_pages)
    if k.shape[1:] != k_pages.shape[1::2]:
        raise ValueError("k, v and the pages must share kv_heads and head_dim")
    _ints(k, torch.int64, slots=slots)
    if slots.shape != k.shape[:1]:
        raise ValueError("slots needs one entry per token")
    p, _ = _cache_problem(0, k.shape[0], 0, k.shape[1], k.shape[2], k_pages.shape[0],
                          k_pages.shape[2], 0, 1, 0, 0, 0, k.dtype, 1.0,
                          (None, k.stride(), v.stride(), None))
    _call(lib.na_cache_write, k.device, p, k.data_ptr(), v.data_ptr(), slots.data_ptr(),
          k_pages.data_ptr(), v_pages.data_ptr())


def cache_attention(q, k_pages, v_pages, page_table, context_lens, cu_new, kernel_size=None,
                    sinks=0, scale=None, max_new=None, max_context=None, out=None, lse=None):
    """Attention of new tokens q [tokens, heads, head_dim] over the cache that already holds
    their keys and values: token t of request r is row cu_new[r] + t, at position
    context_lens[r] + t.  kernel_size None: the whole context.  max_new and max_context, bounds
    of the new tokens and of the whole tokens of any request where the caller knows them, only
    choose how the work is split.  Returns (out, logsumexp [tokens, heads] fp32); rows from
    cu_new[requests] on are left as they were.  A page id outside the pages reads as zeros."""
    lib = _library()
    if q.dim() != 3:
        raise ValueError("expected q [tokens, heads, head_dim]")
    _check_pages(q, k_pages, v_pages)
    kv_heads = k_pages.shape[1]
    if q.shape[2] != k_pages.shape[3]:
        raise ValueError("q and the pages must share head_dim")
    if q.shape[1] != kv_heads and (kv_heads == 0 or q.shape[1] % kv_heads):
        raise ValueError("the heads of q must be a multiple of those of the pages")
    if context_lens.dim() != 1 or page_table.dim() != 2 \
            or page_table.shape[0] != context_lens.shape[0]:
        raise ValueError("expected context_lens [requests] and page_table [requests, max_pages]")
    if cu_new.shape != (context_lens.shape[0] + 1,):
        raise ValueError("cu_new needs one entry more than there are requests")
    out = _like(q) if out is None else out
    if lse is None:
        lse = torch.empty(q.shape[:-1], dtype=torch.float32, device=q.device)
    if out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    _rows(q, out)
    _check_lse(lse, q)
    _ints(q, torch.int32, page_table=page_table, context_lens=context_lens, cu_new=cu_new)
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1])
    p, need = _cache_problem(
        context_lens.shape[0], q.shape[0], q.shape[1], kv_heads, q.shape[2], k_pages.shape[0],
        k_pages.shape[2], page_table.shape[1],
        _WHOLE if kernel_size is None else _count(kernel_size, "kernel_size", 1),
        _count(sinks, "sinks", 0), 0 if max_new is None else _count(max_new, "max_new", 0),
        0 if max_context is None else _count(max_context, "max_context", 0), q.dtype,
        float(scale), (q.stride(), None, None, out.stride()))
    # (the allocator hands it out stream by stream, and to a captured graph from its own pool)
    work = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    _call(lib.na_cache_attention, q.device, p, q.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), page_table.data_ptr(), context_lens.data_ptr(), cu_new.data_ptr(),
          out.data_ptr(), lse.data_ptr(), work.data_ptr() if need else 0, need)
    return out, lse


def cache_step(q, k, v, k_pages, v_pages, page_table, context_lens, new_lens, free_pages,
               kernel_size=None, sinks=0, scale=None, head=None, max_new=None, max_context=None,
               tables=None):
    """One serving step of an attention layer: the tables of the new tokens, their keys and
    values into the pages, and their attention.  q [tokens, heads, head_dim], k and v [tokens,
    kv_heads, head_dim] hold the requests' new tokens one after another.  `tables`: what
    cache_tables returned for this step (the layers of a model share it); None builds it.
    Returns (out, logsumexp, new_head)."""
    if q.dim() != 3 or q.shape[0] != k.shape[0]:
        raise ValueError("q, k and v need the same new tokens")
    if tables is None:
        tables = cache_tables(context_lens, new_lens, page_table, free_pages, k_pages.shape[2],
                              q.shape[0], head)
    cu_new, slots, _, new_head = tables
    cache_write(k, v, slots, k_pages, v_pages)
    out, lse = cache_attention(q, k_pages, v_pages, page_table, context_lens, cu_new, kernel_size,
                               sinks, scale, max_new, max_context)
    return out, lse, new_head
