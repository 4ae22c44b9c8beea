"""Performance cases of the sequence operators: attention over a sliding window and the first
tokens, and the paged cache that serves it (tables, writes, attention of new tokens).

A case names its operator and how a program calls it:

  op = "sink"    attention over the kernel_size nearest earlier tokens and the first `sinks`;
                 call = "forward" (inference: out, logsumexp), "explicit" (a training step that
                 keeps its own graph: out, logsumexp, dq, dk, dv) or "autograd" (out, dq, dk, dv)
  op = "tables"  the page table, slots and positions of a batch of new tokens
  op = "write"   new keys and values into the pages at their slots
  op = "attend"  new tokens against the cache that already holds them
  op = "step"    tables, write and attention of one serving step

Inputs are iid N(0, 1) in the case's type (projected, normalised activations), drawn on the GPU
from the seed; lengths follow from the case alone, so that its work is known without inputs.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
WHOLE = 0  # kernel_size of attention over the whole context


def _sink(name, call, dtype, batch, heads, kv_heads, tokens, head_dim, kernel, sinks,
          ragged=False):
    return {"name": name, "op": "sink", "call": call, "dtype": dtype, "batch": batch,
            "heads": heads, "kv_heads": kv_heads, "tokens": tokens, "head_dim": head_dim,
            "kernel": kernel, "sinks": sinks, "ragged": ragged, "mix": 1}


def _cache(name, op, dtype, requests, heads, kv_heads, head_dim, page, context, new, kernel=WHOLE,
           sinks=0, mix=1):
    """context, new: (fewest, most) tokens of a request before the step and of the step."""
    return {"name": name, "op": op, "dtype": dtype, "requests": requests, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "context_lo": context[0],
            "context_hi": context[1], "new_lo": new[0], "new_hi": new[1], "kernel": kernel,
            "sinks": sinks, "mix": mix}


def listed():
    return [
        # the smallest call: one short sequence, full precision; launch latency
        _sink("sink_small_fp32_fwd", "forward", "fp32", 1, 2, 2, 256, 32, 7, 4),
        # a padded batch of unequal sequences, three query heads to a key head: training
        _sink("sink_ragged_fp16_step", "explicit", "fp16", 3, 6, 2, 1531, 64, 255, 4, True),
        # a sliding-window language model's layer, four query heads to a key head: training
        _sink("sink_bf16_step", "autograd", "bf16", 1, 16, 4, 8192, 128, 512, 4),
        # a long document read at once: inference
        _sink("sink_long_fp16_fwd", "forward", "fp16", 1, 16, 16, 32768, 64, 1023, 16),
        # a decoding server's step: one token for each request
        _cache("tables_decode", "tables", "bf16", 64, 16, 4, 128, 16, (1, 8192), (1, 1)),
        # prompts of many requests admitted at once, odd lengths, some requests idle
        _cache("tables_prompts", "tables", "bf16", 256, 16, 4, 128, 64, (0, 4096), (0, 511)),
        # one token for each request into the cache
        _cache("write_decode", "write", "fp16", 64, 16, 4, 64, 16, (1, 4096), (1, 1)),
        # the tokens of long prompts into the cache
        _cache("write_prompts", "write", "bf16", 16, 16, 8, 128, 64, (0, 1000), (1500, 2500)),
        # a small batch decoding with a window and sinks: a whole step, launch latency
        _cache("step_decode_window_bf16", "step", "bf16", 8, 16, 4, 128, 16, (100, 8192), (1, 1),
               512, 4),
        # a batch decoding over long contexts: the cache is read once
        _cache("attend_decode_long_fp16", "attend", "fp16", 32, 16, 4, 128, 64, (8192, 32768),
               (1, 1)),
        # chunks of long prompts over what is cached of them
        _cache("attend_chunk_bf16", "attend", "bf16", 4, 16, 4, 128, 64, (2048, 8192),
               (512, 2048)),
        # odd chunks in full precision with a window and sinks, one key head
        _cache("attend_chunk_window_fp32", "attend", "fp32", 5, 6, 1, 64, 16, (0, 2000), (1, 257),
               255, 20),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm from lo to hi (lo may be 0)."""
    return int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1


_HEADS = ((1, 1), (2, 2), (4, 1), (4, 4), (6, 2), (8, 8), (10, 2), (16, 4), (16, 16))
_LARGEST = 2.6e11  # products of the largest listed case, in 16-bit terms
_LARGEST_BYTES = 1.0e9
_LARGEST_PLAIN = 2.2e9  # (query, key) pairs of all heads that a dense form would visit


def draw(rng):
    while True:
        op = rng.choice(("sink", "sink", "sink", "tables", "write", "attend", "attend", "step"))
        dtype = rng.choice(("fp16", "fp16", "bf16", "bf16", "fp32"))
        heads, kv_heads = rng.choice(_HEADS)
        head_dim = rng.choice((32, 64, 64, 128, 128))
        sinks = rng.choice((0, 1, 4, 4, 16, 33))
        if op == "sink":
            case = _sink("", rng.choice(("forward", "explicit", "autograd")), dtype,
                         rng.choice((1, 1, 2, 3, 5)), heads, kv_heads,
                         max(1, _log_int(rng, 100, 32768)), head_dim,
                         max(1, _log_int(rng, 6, 1500)), sinks, rng.random() < 0.4)
        else:
            kind = rng.choice(("decode", "chunk"))
            requests = max(1, _log_int(rng, 1, 256 if op in ("tables", "write") else 48))
            new = (1, 1) if kind == "decode" else (rng.choice((0, 1)), _log_int(rng, 16, 2048))
            hi = _log_int(rng, 64, 32768 if kind == "decode" else 8192)
            kernel = rng.choice((WHOLE, max(1, _log_int(rng, 30, 2048))))
            case = _cache("", op, dtype, requests, heads, kv_heads, head_dim,
                          rng.choice((16, 16, 32, 64, 128)), (0 if kind == "chunk" else hi // 4, hi),
                          new, kernel, sinks if kernel != WHOLE else 0)
        case["mix"] = rng.randrange(1 << 30)
        del case["name"]
        w = work(case)
        dense = 0
        if op in ("attend", "step"):
            ctx, new = _lens(case)
            dense = case["requests"] * heads * max(new) * max(c + n for c, n in zip(ctx, new))
        elif op == "sink":
            case_rows = case["batch"] * heads * case["tokens"]
            dense = case_rows * min(2 * case["kernel"] + sinks, case["tokens"] + sinks)
        # full precision has a sixteenth of the 16-bit rate; a dense form has to fit the card
        if (0 < w["bytes"] <= _LARGEST_BYTES and dense <= _LARGEST_PLAIN
                and w["flops"] * (16 if dtype == "fp32" else 1) <= _LARGEST
                and (op == "sink" or sum(_lens(case)[1]) > 0)):
            return case


def _lens(case):
    """Tokens of each request before the step, and of the step."""
    rng = random.Random(case["mix"])
    ctx = [_log_int(rng, case["context_lo"], case["context_hi"]) for _ in range(case["requests"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["requests"])]
    return ctx, new


def _lengths(case):
    """Valid tokens of each sequence of a padded batch (the longest fills it)."""
    rng = random.Random(case["mix"])
    n = case["tokens"]
    return [n if b == 0 else rng.randint(0, n) for b in range(case["batch"])]


def _visible(pos, kernel, sinks):
    """Keys that a token at `pos` attends to."""
    near = min(pos + 1, kernel)
    return near + min(max(pos + 1 - kernel, 0), sinks)


def work(case):
    row = case["head_dim"] * BYTES[case["dtype"]]
    if case["op"] == "sink":
        lens = _lengths(case) if case["ragged"] else [case["tokens"]] * case["batch"]
        tokens = case["batch"] * case["tokens"]
        pairs = case["heads"] * sum(_visible(p, case["kernel"], case["sinks"])
                                    for n in lens for p in range(n))
        # read q, k, v, write out and the fp32 logsumexp; two products a pair
        q, kv = tokens * case["heads"] * row, tokens * case["kv_heads"] * row
        size = 2 * q + 2 * kv + tokens * case["heads"] * 4
        flops = 4 * case["head_dim"] * pairs
        if case["call"] != "forward":
            # a step: read dout too, write dq, dk, dv; five more products a pair
            size += 2 * q + 2 * kv
            flops += 10 * case["head_dim"] * pairs
        return {"bytes": size, "flops": flops}
    ctx, new = _lens(case)
    total, page = sum(new), case["page"]
    size = flops = 0
    if case["op"] in ("tables", "step"):
        # lengths, the pages handed out (read and written), offsets, slots and positions
        pages = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(ctx, new))
        size += case["requests"] * 12 + pages * 8 + total * 12
    if case["op"] in ("write", "step"):
        size += 4 * total * case["kv_heads"] * row + total * 8
    if case["op"] in ("attend", "step"):
        kernel = case["kernel"] or (1 << 31) - 1
        keys = pairs = 0
        for c, n in zip(ctx, new):
            if n:
                # one request's tokens share their keys: the first one's and the tokens between
                keys += _visible(c, kernel, case["sinks"]) + n - 1
                pairs += sum(_visible(p, kernel, case["sinks"]) for p in range(c, c + n))
        size += 2 * total * case["heads"] * row + total * case["heads"] * 4
        size += 2 * keys * case["kv_heads"] * row
        flops += 4 * case["head_dim"] * case["heads"] * pairs
    return {"bytes": size, "flops": flops}


# ---------------------------------------------------------------- inputs

def _randn(gen, shape, case):
    return torch.randn(shape, generator=gen, device="cuda").to(DTYPES[case["dtype"]])


def _sink_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, d = case["tokens"], case["head_dim"]
    heads = [case["heads"], case["kv_heads"], case["kv_heads"], case["heads"]]
    ts = [_randn(gen, (case["batch"], h, n, d), case)
          for h in heads[:3 if case["call"] == "forward" else 4]]
    lens = None
    if case["ragged"]:
        lens = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    return ts, lens


def _cache_inputs(case, seed):
    """A server's state before a step: pages in any order, the free ones, and the new tokens."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ctx, new = _lens(case)
    page, need = case["page"], max(c + n for c, n in zip(*_lens(case)))
    held = [-(-c // page) for c in ctx]
    after = [-(-(c + n) // page) for c, n in zip(ctx, new)]
    pool = sum(after) + 3
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32).cpu()
    most = max(1, -(-need // page))
    table = torch.full((case["requests"], most), -1, dtype=torch.int32)
    used = 0
    for r, h in enumerate(held):
        table[r, :h] = order[used:used + h]
        used += h
    free = order[used:]
    state = {"context_lens": torch.tensor(ctx, dtype=torch.int32, device="cuda"),
             "new_lens": torch.tensor(new, dtype=torch.int32, device="cuda"),
             "free_pages": free.cuda(), "block_table": table.cuda(), "tokens": sum(new),
             "max_new": max(new), "max_context": need}
    if case["op"] == "tables":
        return state
    pages = (pool, case["kv_heads"], page, case["head_dim"])
    state["k_pages"], state["v_pages"] = (_randn(gen, pages, case) for _ in range(2))
    if case["op"] == "attend" or case["op"] == "write":
        # the tables of the step, as cache_tables leaves them
        state.update(_plain_tables(state, page))
    rows = (sum(new), case["kv_heads"], case["head_dim"])
    if case["op"] in ("write", "step"):
        state["k"], state["v"] = (_randn(gen, rows, case) for _ in range(2))
    if case["op"] in ("attend", "step"):
        state["q"] = _randn(gen, (sum(new), case["heads"], case["head_dim"]), case)
    return state


def prepare(case, seed):
    state = {"op": case["op"], "kernel": case["kernel"], "sinks": case["sinks"]}
    if case["op"] == "sink":
        ts, state["lengths"] = _sink_inputs(case, seed)
        state["call"] = case["call"]
        state.update(zip(("q", "k", "v", "dout"), ts))
        if case["call"] == "autograd":
            for name in ("q", "k", "v"):
                state[name].requires_grad_(True)
        return state
    state["page"] = case["page"]
    state.update(_cache_inputs(case, seed))
    return state


# ---------------------------------------------------------------- plain forms

def _plain_sink(s):
    """Blocks of queries against the keys that any of them sees, in 32 bits."""
    q, k, v = (s[n].detach().float() for n in ("q", "k", "v"))
    B, H, N, D = q.shape
    kv, kernel, sinks = k.shape[1], s["kernel"], min(s["sinks"], N)
    G, scale = H // kv, 1.0 / math.sqrt(D)
    size = min(max(64, min(kernel, 1024)), N)
    blocks = -(-N // size)
    back = min(kernel - 1, N - 1)
    dev = q.device
    pos = torch.arange(blocks * size, device=dev).reshape(blocks, size)
    # a block's keys: the first tokens, then its window (the first tokens counted once)
    near = (torch.arange(blocks, device=dev) * size)[:, None] + torch.arange(-back, size,
                                                                             device=dev)
    first = torch.arange(sinks, device=dev).expand(blocks, sinks)
    key = torch.cat([first, near], 1)
    extra = torch.arange(key.shape[1], device=dev) < sinks
    i, j = pos[:, :, None], key[:, None, :]
    inside = (j <= i) & (i - j < kernel)
    seen = torch.where(extra, (j <= i) & ~inside, inside & (j >= 0)) & (i < N)
    lens = s["lengths"] if s["lengths"] is not None else torch.full((B,), N, device=dev)
    at = key.clamp(0, N - 1)
    rows = pos.clamp(max=N - 1)

    def heads(x):  # [B, H, N, D] -> [B, kv, blocks, G size, D]
        x = x.reshape(B, kv, G, N, D)[:, :, :, rows]
        return x.permute(0, 1, 3, 2, 4, 5).reshape(B, kv, blocks, G * size, D)

    def back_to(x, *tail):  # [B, kv, blocks, G size, ..] -> [B, H, N, ..]
        x = x.reshape(B, kv, blocks, G, size, *tail).transpose(2, 3)
        return x.reshape(B, H, blocks * size, *tail)[:, :, :N]

    mask = seen[None] & (i < lens[:, None, None, None]) & (j < lens[:, None, None, None])
    mask = mask[:, None, :, None].expand(B, 1, blocks, G, size, key.shape[1])
    mask = mask.reshape(B, 1, blocks, G * size, key.shape[1])
    qb, kb, vb = heads(q), k[:, :, at], v[:, :, at]
    p = torch.matmul(qb, kb.transpose(-1, -2)).mul_(scale).masked_fill_(~mask, -math.inf)
    top = p.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top).masked_fill(total == 0, -math.inf)
    p.div_(total.clamp(min=1e-38))
    out = torch.matmul(p, vb)
    res = [back_to(out, D).to(s["q"].dtype)]
    if s["call"] != "autograd":
        res.append(back_to(lse.squeeze(-1)))
    if s["call"] == "forward":
        return tuple(res)
    g = heads(s["dout"].float())
    delta = (g * out).sum(-1, keepdim=True)
    dv = torch.matmul(p.transpose(-1, -2), g)
    p.mul_(torch.matmul(g, vb.transpose(-1, -2)).sub_(delta)).mul_(scale)
    dq = back_to(torch.matmul(p, kb), D)
    dk = torch.matmul(p.transpose(-1, -2), qb)
    at = at.reshape(-1)
    grads = [torch.zeros(B, kv, N, D, device=dev).index_add_(2, at, x.reshape(B, kv, -1, D))
             for x in (dk, dv)]
    return tuple(res) + tuple(x.to(s["q"].dtype) for x in [dq] + grads)


def _plain_tables(s, page):
    """cu_new, slots, positions and the page table; the new pages are the first free ones."""
    c, n, table = s["context_lens"].long(), s["new_lens"].long(), s["block_table"]
    cu = torch.cat([n.new_zeros(1), n.cumsum(0)])
    held, after = (c + page - 1) // page, (c + n + page - 1) // page
    base = (after - held).cumsum(0) - (after - held)
    col = torch.arange(table.shape[1], device=table.device)
    fresh = (col >= held[:, None]) & (col < after[:, None])
    taken = (base[:, None] + col - held[:, None]).clamp(0, s["free_pages"].numel() - 1)
    table.copy_(torch.where(fresh, s["free_pages"][taken], table))
    i = torch.arange(s["tokens"], device=table.device)
    r = torch.searchsorted(cu[1:], i, right=True)
    pos = c[r] + i - cu[r]
    slots = table[r, pos // page].long() * page + pos % page
    return {"cu_new": cu.int(), "slots": slots, "positions": pos.int(), "block_table": table,
            "head": (after - held).sum().int().reshape(1)}


def _plain_write(s):
    page = s["page"]
    for pages, rows in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        pages[s["slots"] // page, :, s["slots"] % page] = rows


def _plain_attend(s):
    """Every request padded to the longest context and the most new tokens, in 32 bits."""
    q, table, page = s["q"].float(), s["block_table"], s["page"]
    T, H, D = q.shape
    kv, kernel = s["k_pages"].shape[1], s["kernel"] or (1 << 31) - 1
    G, R, most, span = H // kv, table.shape[0], s["max_new"], s["max_context"]
    dev = q.device
    c, cu = s["context_lens"].long(), s["cu_new"].long()
    n = cu[1:] - cu[:-1]
    t = torch.arange(most, device=dev)
    tok = (cu[:-1, None] + t).clamp(max=T - 1)  # [R, most]
    live = t < n[:, None]
    key = torch.arange(span, device=dev)
    ids = table[:, key // page].clamp(min=0).long()

    def cached(pages):  # [R, kv, span, D]
        return pages[ids, :, key % page].permute(0, 2, 1, 3).float()

    qb = q[tok].reshape(R, most, kv, G, D).permute(0, 2, 3, 1, 4).reshape(R, kv, G * most, D)
    p = torch.matmul(qb, cached(s["k_pages"]).transpose(-1, -2)).mul_(1.0 / math.sqrt(D))
    i = (c[:, None] + t)[:, :, None]
    seen = (key <= i) & ((i - key < kernel) | (key < s["sinks"])) & live[:, :, None]
    p = p.reshape(R, kv, G, most, span).masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1)
    # values behind a request's own tokens are nothing of its
    values = cached(s["v_pages"]).masked_fill_((key >= (c + n)[:, None])[:, None, :, None], 0.0)
    out = torch.matmul(p.reshape(R, kv, G * most, span), values).reshape(R, kv, G, most, D)
    out = out / total.clamp(min=1e-38)
    where = torch.searchsorted(cu[1:], torch.arange(T, device=dev), right=True)
    at = torch.arange(T, device=dev) - cu[where]
    out = out.permute(0, 3, 1, 2, 4)[where, at].reshape(T, H, D)
    lse = lse.permute(0, 3, 1, 2)[where, at].reshape(T, H)
    return out.to(s["q"].dtype), lse


def _plain(s):
    if s["op"] == "sink":
        return _plain_sink(s)
    if s["op"] in ("tables", "step"):
        t = _plain_tables(s, s["page"])
        if s["op"] == "tables":
            return t["cu_new"], t["slots"], t["positions"], t["head"], t["block_table"]
        s = {**s, **t}
    if s["op"] in ("write", "step"):
        _plain_write(s)
        if s["op"] == "write":
            return s["k_pages"], s["v_pages"]
    out = _plain_attend(s)
    if s["op"] == "step":
        return out + (t["head"], s["block_table"], s["k_pages"], s["v_pages"])
    return out


def run(s):
    if not own:
        return _plain(s)
    import paper_2403_04690_amd as na

    if s["op"] == "sink":
        q, k, v, ks, sinks, lens = (s[n] for n in ("q", "k", "v", "kernel", "sinks", "lengths"))
        if s["call"] == "autograd":
            out = na.sink_attention(q, k, v, ks, sinks, lengths=lens)
            return (out.detach(),) + torch.autograd.grad(out, (q, k, v), s["dout"])
        out, lse = na.sink_forward(q, k, v, ks, sinks, lengths=lens)
        if s["call"] == "forward":
            return out, lse
        return (out, lse) + na.sink_backward(q, k, v, out, lse, s["dout"], ks, sinks,
                                             lengths=lens)
    ks = s["kernel"] or None
    if s["op"] == "tables":
        return na.cache_tables(s["context_lens"], s["new_lens"], s["block_table"],
                               s["free_pages"], s["page"], s["tokens"]) + (s["block_table"],)
    if s["op"] == "write":
        na.cache_write(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"])
        return s["k_pages"], s["v_pages"]
    if s["op"] == "attend":
        return na.cache_attention(s["q"], s["k_pages"], s["v_pages"], s["block_table"],
                                  s["context_lens"], s["cu_new"], ks, s["sinks"],
                                  max_new=s["max_new"], max_context=s["max_context"])
    out, lse, head = na.cache_step(s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"],
                                   s["block_table"], s["context_lens"], s["new_lens"],
                                   s["free_pages"], ks, s["sinks"], max_new=s["max_new"],
                                   max_context=s["max_context"])
    return out, lse, head, s["block_table"], s["k_pages"], s["v_pages"]


# ---------------------------------------------------------------- 64 bits

def _attention64(q, k, v, i, j, kernel, sinks, g=None):
    """Rows q at positions i against k, v at positions j, all heads of one key head: out,
    logsumexp and, with g, the gradients."""
    scale = q.shape[-1] ** -0.5
    dist = i[:, None] - j[None, :]
    hide = (dist < 0) | ((dist >= kernel) & (j[None, :] >= sinks))
    a = (q @ k.T * scale).masked_fill_(hide, -math.inf)
    lse = torch.logsumexp(a, -1)
    a = torch.exp_(a.sub_(lse[:, None]))
    out = a @ v
    if g is None:
        return out, lse
    da = a * (g @ v.T - (g * out).sum(-1, keepdim=True)) * scale
    return out, lse, da @ k, da.T @ q, a.T @ g


def _exact_sink(case, seed):
    ts, _ = _sink_inputs(case, seed)
    q, k, v = (x.double() for x in ts[:3])
    g = ts[3].double() if len(ts) > 3 else None
    B, H, N, D = q.shape
    kv, step = k.shape[1], 2048
    lens = _lengths(case) if case["ragged"] else [N] * B
    out, dq = torch.zeros_like(q), torch.zeros_like(q)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(H):
            c = h // (H // kv)
            for lo in range(0, lens[b], step):
                hi = min(lo + step, lens[b])
                from_ = max(0, lo - case["kernel"] + 1)
                few = min(case["sinks"], from_)
                keys = torch.cat([torch.arange(few), torch.arange(from_, hi)]).cuda()
                rows = torch.arange(lo, hi, device="cuda")
                r = _attention64(q[b, h, lo:hi], k[b, c, keys], v[b, c, keys], rows, keys,
                                 case["kernel"], case["sinks"],
                                 None if g is None else g[b, h, lo:hi])
                out[b, h, lo:hi], lse[b, h, lo:hi] = r[:2]
                if g is not None:
                    dq[b, h, lo:hi] = r[2]
                    dk[b, c].index_add_(0, keys, r[3])
                    dv[b, c].index_add_(0, keys, r[4])
    res = (out,) if case["call"] == "autograd" else (out, lse)
    return res if g is None else res + (dq, dk, dv)


def exact(case, seed):
    if case["op"] == "sink":
        return _exact_sink(case, seed)
    if case["op"] == "tables":
        return None  # whole numbers
    s = _cache_inputs(case, seed)
    ctx, new = _lens(case)
    page, G = case["page"], case["heads"] // case["kv_heads"]
    table, free, used = s["block_table"].cpu().tolist(), s["free_pages"].cpu().tolist(), 0
    T, H, D = s["tokens"], case["heads"], case["head_dim"]
    out = torch.zeros(T, H, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    k_pages, v_pages = (s[n].double() for n in ("k_pages", "v_pages"))
    at = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        if case["op"] == "step":
            for x in range(-(-c // page), -(-(c + n) // page)):
                table[r][x] = free[used]
                used += 1
        ids = torch.tensor(table[r][:-(-(c + n) // page)], device="cuda")
        if case["op"] in ("step", "write"):
            p = torch.arange(c, c + n, device="cuda")
            k_pages[ids[p // page], :, p % page] = s["k"][at:at + n].double()
            v_pages[ids[p // page], :, p % page] = s["v"][at:at + n].double()
        if case["op"] == "write":
            at += n
            continue
        j = torch.arange(c + n, device="cuda")
        rows = torch.arange(c, c + n, device="cuda").repeat_interleave(G)
        for h in range(case["kv_heads"]):
            kk, vv = (x[ids, h].reshape(-1, D)[:c + n] for x in (k_pages, v_pages))
            q = s["q"][at:at + n, h * G:(h + 1) * G].double().reshape(n * G, D)
            o, e = _attention64(q, kk, vv, rows, j, case["kernel"] or (1 << 31) - 1,
                                case["sinks"])
            out[at:at + n, h * G:(h + 1) * G] = o.reshape(n, G, D)
            lse[at:at + n, h * G:(h + 1) * G] = e.reshape(n, G)
        at += n
    if case["op"] == "write":
        return k_pages, v_pages
    return (out, lse) if case["op"] == "attend" else (out, lse, None, None, k_pages, v_pages)
