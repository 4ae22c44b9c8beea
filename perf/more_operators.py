"""Performance cases of the cache operators for long contexts: attention of a batch whose requests
share long prefixes, the attention weight that cached keys gather, and the eviction of the keys
that gathered least.

A case names its operator:

  op = "shared"   new tokens against the cache; groups of requests share their first tokens
  op = "weights"  the attention weights of new tokens added up for every key of the cache
  op = "evict"    requests cut back to `budget` tokens a key/value head: the first, the last and
                  the heaviest of the others, which stay where they are or fill the places of
                  the ones that go

Inputs are iid N(0, 1) in the case's type (projected, normalised activations), drawn on the GPU
from the seed; gathered weights spread over orders of magnitude, with ties.  Lengths follow from
the case alone, so that its work is known without inputs.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}
WHOLE = 0  # kernel_size of attention over the whole context
_FAR = (1 << 31) - 1


def _shared(name, dtype, requests, groups, heads, kv_heads, head_dim, page, shared, context, new,
            kernel=WHOLE, sinks=0, mix=1):
    """shared, context, new: (fewest, most) tokens that a group shares, that a request has cached
    of its own, and that it gets."""
    return {"name": name, "op": "shared", "dtype": dtype, "requests": requests, "groups": groups,
            "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
            "shared_lo": shared[0], "shared_hi": shared[1], "context_lo": context[0],
            "context_hi": context[1], "new_lo": new[0], "new_hi": new[1], "kernel": kernel,
            "sinks": sinks, "mix": mix}


def _weights(name, dtype, requests, heads, kv_heads, head_dim, page, context, new, kernel=WHOLE,
             sinks=0, first=(0, 0), mix=1):
    """first: (fewest, most) of a request's first tokens whose weight nobody asks for."""
    return {"name": name, "op": "weights", "dtype": dtype, "requests": requests, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "context_lo": context[0],
            "context_hi": context[1], "new_lo": new[0], "new_hi": new[1], "kernel": kernel,
            "sinks": sinks, "first_lo": first[0], "first_hi": first[1], "mix": mix}


def _evict(name, dtype, requests, kv_heads, head_dim, page, context, budget, recent, first=(0, 0),
           mix=1):
    return {"name": name, "op": "evict", "dtype": dtype, "requests": requests,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "context_lo": context[0],
            "context_hi": context[1], "budget": budget, "recent": recent, "first_lo": first[0],
            "first_hi": first[1], "mix": mix}


def listed():
    return [
        # the smallest call: a few requests behind a short common prompt, full precision
        _shared("shared_small_fp32", "fp32", 4, 1, 2, 2, 32, 16, (300, 300), (1, 60), (1, 1)),
        # a decoding server whose requests all begin with one long system prompt
        _shared("shared_decode_bf16", "bf16", 64, 1, 16, 4, 128, 64, (8192, 8192), (16, 1024),
                (1, 1)),
        # several prompts, a few proposed tokens a request, a long window; odd sizes
        _shared("shared_groups_fp16", "fp16", 45, 3, 6, 2, 64, 16, (1000, 9000), (0, 700), (1, 5),
                6001, 20),
        # new prompts admitted behind a common one: chunks of a prefill
        _shared("shared_prompts_bf16", "bf16", 16, 2, 16, 4, 128, 64, (4096, 8192), (0, 100),
                (64, 300), mix=4),
        # the smallest call: launch latency
        _weights("weights_small_fp32", "fp32", 3, 2, 2, 32, 16, (10, 200), (1, 1)),
        # a batch decoding over long contexts: the keys are read once
        _weights("weights_decode_bf16", "bf16", 32, 16, 4, 128, 64, (8192, 32768), (1, 1)),
        # the tokens of odd chunks of prompts, windowed, their first tokens kept anyway
        _weights("weights_window_fp16", "fp16", 7, 6, 2, 64, 16, (0, 3000), (1, 400), 1023, 16,
                 (0, 40)),
        # chunks of long prompts over what is cached of them
        _weights("weights_chunk_bf16", "bf16", 4, 16, 4, 128, 64, (2048, 8192), (512, 2048)),
        # the smallest call: a handful of tokens over a small budget
        _evict("evict_small_fp32", "fp32", 3, 2, 32, 16, (100, 300), 128, 16),
        # a decoding server trims what its requests gained over the last steps
        _evict("evict_decode_bf16", "bf16", 64, 4, 128, 64, (2049, 2304), 2048, 256, (4, 4)),
        # odd lengths and budget; some requests are below it and stay as they are
        _evict("evict_ragged_fp16", "fp16", 37, 3, 64, 16, (0, 5000), 777, 100, (0, 200)),
        # long prompts just read, cut down before decoding begins
        _evict("evict_prompts_bf16", "bf16", 8, 8, 128, 64, (8192, 32768), 4096, 512, (16, 16)),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm from lo to hi (lo may be 0)."""
    return int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1


_HEADS = ((1, 1), (2, 2), (4, 1), (4, 4), (6, 2), (8, 8), (10, 2), (16, 4))
_LARGEST = 1.0e11  # products of the largest listed case, in 16-bit terms
_LARGEST_BYTES = 8.0e8
_LARGEST_PLAIN = 1.2e9  # (query, key) pairs of all heads that a dense form visits
_LARGEST_GATHER = 4.0e9  # bytes of keys that a dense form gathers in 32 bits


def draw(rng):
    while True:
        op = rng.choice(("shared", "weights", "evict"))
        dtype = rng.choice(("fp16", "fp16", "bf16", "bf16", "fp32"))
        heads, kv_heads = rng.choice(_HEADS)
        head_dim = rng.choice((32, 64, 64, 128, 128))
        page = rng.choice((16, 16, 32, 64, 128))
        kernel = rng.choice((WHOLE, WHOLE, max(1, _log_int(rng, 100, 8192))))
        sinks = rng.choice((0, 1, 4, 16, 33)) if kernel != WHOLE else 0
        kind = rng.choice(("decode", "decode", "few", "chunk"))
        new = {"decode": (1, 1), "few": (0, 8), "chunk": (0, _log_int(rng, 16, 1500))}[kind]
        if op == "shared":
            requests = max(2, _log_int(rng, 2, 100))
            hi = _log_int(rng, 100, 32768)
            case = _shared("", dtype, requests, rng.randint(1, min(5, requests)), heads, kv_heads,
                           head_dim, page, (hi // 4, hi), (0, _log_int(rng, 16, 2048)), new,
                           kernel, sinks)
        elif op == "weights":
            requests = max(1, _log_int(rng, 1, 64))
            hi = _log_int(rng, 64, 32768)
            case = _weights("", dtype, requests, heads, kv_heads, head_dim, page, (hi // 8, hi),
                            new, kernel, sinks, (0, rng.choice((0, 0, 4, 100))))
        else:
            requests = max(1, _log_int(rng, 1, 128))
            hi = _log_int(rng, 64, 32768)
            budget = max(1, _log_int(rng, 16, 4096))
            case = _evict("", dtype, requests, kv_heads, head_dim, page, (hi // 8, hi), budget,
                          int(budget * rng.choice((0, 0.1, 0.5, 1))),
                          (0, rng.choice((0, 4, 100))))
        case["mix"] = rng.randrange(1 << 30)
        del case["name"]
        w = work(case)
        dense = gather = 0
        if op == "evict":
            ctx, _ = _evict_lens(case)
            # (the kept rows, gathered as they are; sorted weights)
            gather = 16 * case["requests"] * kv_heads * max(ctx) \
                + 4 * case["requests"] * kv_heads * min(case["budget"], max(ctx)) * head_dim
            some = max(ctx) > case["budget"]
        else:
            ctx, new_lens = _lens(case)[:2]
            span = max(c + n for c, n in zip(ctx, new_lens))
            dense = requests * heads * max(new_lens) * span
            gather = 8 * requests * kv_heads * span * head_dim
            some = sum(new_lens) > 0
        # full precision has a sixteenth of the 16-bit rate; a dense form has to fit the card
        if (some and 0 < w["bytes"] <= _LARGEST_BYTES and dense <= _LARGEST_PLAIN
                and gather <= _LARGEST_GATHER
                and w["flops"] * (16 if dtype == "fp32" else 1) <= _LARGEST):
            return case


def _lens(case):
    """Cached and new tokens of each request; of a "shared" case also the groups' offsets and the
    tokens that each shares (part of its requests' cached ones)."""
    rng = random.Random(case["mix"])
    R = case["requests"]
    ctx = [_log_int(rng, case["context_lo"], case["context_hi"]) for _ in range(R)]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(R)]
    if case["op"] != "shared":
        return ctx, new
    cuts = sorted(rng.randint(0, R) for _ in range(case["groups"] - 1))
    cu = [0] + cuts + [R]
    shared = [_log_int(rng, case["shared_lo"], case["shared_hi"]) for _ in range(case["groups"])]
    for g in range(case["groups"]):
        for r in range(cu[g], cu[g + 1]):
            ctx[r] += shared[g]
    return ctx, new, cu, shared


def _evict_lens(case):
    """Cached tokens of each request, and how many of the first of them stay."""
    rng = random.Random(case["mix"])
    R = case["requests"]
    ctx = [_log_int(rng, case["context_lo"], case["context_hi"]) for _ in range(R)]
    return ctx, [rng.randint(case["first_lo"], case["first_hi"]) for _ in range(R)]


def _first_lens(case):
    rng = random.Random(case["mix"] + 1)
    return [rng.randint(case["first_lo"], case["first_hi"]) for _ in range(case["requests"])]


def _visible(pos, kernel, sinks):
    """Keys that a token at `pos` attends to."""
    near = min(pos + 1, kernel)
    return near + min(max(pos + 1 - kernel, 0), sinks)


def _visible_from(pos, kernel, sinks, first):
    """Of those, the ones at or behind position `first`."""
    lo = max(pos - kernel + 1, 0)
    near = max(0, pos + 1 - max(lo, first))
    return near + max(0, min(lo, sinks) - first)


def work(case):
    row = case["head_dim"] * BYTES[case["dtype"]]
    page = case["page"]
    if case["op"] == "evict":
        ctx, first = _evict_lens(case)
        size = 0
        for n, f in zip(ctx, first):
            kept = min(n, case["budget"])
            # weights read and the kept ones written, the kept indices, and of requests over the
            # budget the rows of K and V that move, read and written: the last tokens, and those
            # of the heaviest that lie behind the places of the others (as many as with weights
            # that do not depend on the place)
            size += case["kv_heads"] * (4 * n + 4 * kept + 4 * case["budget"])
            if n > case["budget"]:
                f = min(f, case["budget"])
                last = min(case["recent"], case["budget"] - f)
                heavy = case["budget"] - f - last
                moved = last + heavy * (n - case["budget"]) / (n - f - last)
                size += case["kv_heads"] * 4 * int(moved) * row
                size += 8 * (-(-n // page) - -(-case["budget"] // page))
        return {"bytes": size + 12 * case["requests"], "flops": 0}
    kernel = case["kernel"] or _FAR
    ctx, new = _lens(case)[:2]
    total = sum(new)
    size = total * case["heads"] * (row + 4) + 12 * case["requests"]
    pairs = keys = 0
    if case["op"] == "weights":
        for c, n, f in zip(ctx, new, _first_lens(case)):
            if n:
                keys += _visible_from(c, kernel, case["sinks"], f) + max(0, min(n - 1, c + n - f))
                pairs += sum(_visible_from(p, kernel, case["sinks"], f) for p in range(c, c + n))
        size += keys * case["kv_heads"] * (row + 8)
        return {"bytes": size, "flops": 2 * case["head_dim"] * case["heads"] * pairs}
    cu, shared = _lens(case)[2:]
    for g, n in enumerate(shared):
        rows = [(ctx[r], new[r]) for r in range(cu[g], cu[g + 1]) if new[r]]
        if not rows:
            continue
        # the shared keys that the least advanced row sees, once, and each request's own
        least = min(c for c, _ in rows)
        keys += n - max(0, min(n, least - kernel + 1) - case["sinks"])
        for c, m in rows:
            keys += max(0, min(c - n, kernel)) + m
            pairs += sum(_visible(p, kernel, case["sinks"]) for p in range(c, c + m))
    size += total * case["heads"] * row + 2 * keys * case["kv_heads"] * row
    return {"bytes": size, "flops": 4 * case["head_dim"] * case["heads"] * pairs}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, shape, case):
    return torch.randn(shape, generator=gen, device="cuda").to(DTYPES[case["dtype"]])


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _offsets(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _pages(gen, case, held):
    """A table with held[r] pages of request r, in any order over a pool; the free ones."""
    pool = sum(held) + 3
    order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32).cpu()
    table = torch.full((case["requests"], max(1, max(held))), -1, dtype=torch.int32)
    used = 0
    for r, h in enumerate(held):
        table[r, :h] = order[used:used + h]
        used += h
    return pool, table, order


def _shared_inputs(case, seed):
    gen, page = _gen(seed), case["page"]
    ctx, new, cu, shared = _lens(case)
    # whole shared pages are the same ones; the page in which the shared tokens end is each
    # request's own, with a copy of its shared rows
    whole = [0] * case["requests"]
    for g, n in enumerate(shared):
        for r in range(cu[g], cu[g + 1]):
            whole[r] = n // page if r > cu[g] else 0
    held = [-(-(c + n) // page) for c, n in zip(ctx, new)]
    pool, table, order = _pages(gen, case, [h - w for h, w in zip(held, whole)])
    full = torch.full((case["requests"], max(1, max(held))), -1, dtype=torch.int32)
    for g in range(case["groups"]):
        for r in range(cu[g], cu[g + 1]):
            full[r, :whole[r]] = full[cu[g], :whole[r]]
            full[r, whole[r]:held[r]] = table[r, :held[r] - whole[r]]
    k_pages, v_pages = (_randn(gen, (pool, case["kv_heads"], page, case["head_dim"]), case)
                        for _ in range(2))
    for g, n in enumerate(shared):
        rest, many = n % page, cu[g + 1] - cu[g]
        if rest and many > 1:
            ids = full[cu[g]:cu[g + 1], n // page].long().cuda()
            for pages in (k_pages, v_pages):
                pages[ids[1:], :, :rest] = pages[ids[:1], :, :rest]
    return {"q": _randn(gen, (sum(new), case["heads"], case["head_dim"]), case),
            "k_pages": k_pages, "v_pages": v_pages, "page_table": full.cuda(),
            "context_lens": _int32(ctx), "cu_new": _int32(_offsets(new)),
            "cu_groups": _int32(cu), "shared_lens": _int32(shared), "max_new": max(new),
            "max_shared": max(shared), "requests_of_group": max(b - a for a, b in zip(cu, cu[1:])),
            "max_own": max(ctx[r] + new[r] - shared[g] for g in range(case["groups"])
                           for r in range(cu[g], cu[g + 1]))}


def _weights_inputs(case, seed):
    gen, page = _gen(seed), case["page"]
    ctx, new = _lens(case)
    held = [-(-(c + n) // page) for c, n in zip(ctx, new)]
    pool, table, _ = _pages(gen, case, held)
    s = {"q": _randn(gen, (sum(new), case["heads"], case["head_dim"]), case),
         "k_pages": _randn(gen, (pool, case["kv_heads"], page, case["head_dim"]), case),
         "page_table": table.cuda(), "context_lens": _int32(ctx), "cu_new": _int32(_offsets(new)),
         "first": _int32(_first_lens(case)) if case["first_hi"] else None, "max_new": max(new),
         "max_context": max(c + n for c, n in zip(ctx, new)), "page": page,
         "kernel": case["kernel"], "sinks": case["sinks"]}
    # what a few steps before gathered
    room = (case["requests"], case["kv_heads"], table.shape[1] * page)
    rows = sum(new) / case["requests"] * case["heads"] / case["kv_heads"]
    s["weights"] = torch.rand(room, generator=gen, device="cuda").pow_(4)
    s["weights"].mul_(8 * rows / s["max_context"])
    # the logsumexp that the step's attention returned
    s["lse"] = _by_token(s, torch.logsumexp(_scores(s), -1)).contiguous()
    return s


def _evict_inputs(case, seed):
    gen, page = _gen(seed), case["page"]
    ctx, first = _evict_lens(case)
    pool, table, order = _pages(gen, case, [-(-c // page) for c in ctx])
    room = (case["requests"], case["kv_heads"], table.shape[1] * page)
    # weights over orders of magnitude; one in sixteen never gathered any
    w = torch.randn(room, generator=gen, device="cuda").mul_(3).exp_()
    w.mul_(torch.rand(room, generator=gen, device="cuda") > 1 / 16)
    w.masked_fill_(torch.arange(room[2], device="cuda") >= _int32(ctx)[:, None, None], 0.0)
    rows = (pool, case["kv_heads"], page, case["head_dim"])
    return {"weights": w, "k_pages": _randn(gen, rows, case), "v_pages": _randn(gen, rows, case),
            "page_table": table.cuda(), "context_lens": _int32(ctx), "free_pages": order.cuda(),
            "head": _int32([sum(-(-c // page) for c in ctx)]), "budget": case["budget"],
            "recent": case["recent"], "first": _int32(first) if case["first_hi"] else None,
            "page": page}


def prepare(case, seed):
    make = {"shared": _shared_inputs, "weights": _weights_inputs, "evict": _evict_inputs}
    state = make[case["op"]](case, seed)
    state["op"] = case["op"]
    if case["op"] == "shared":
        state.update(kernel=case["kernel"], sinks=case["sinks"], page=case["page"])
    return state


# ---------------------------------------------------------------- plain forms

def _rows(s):
    """q, padded to the most new tokens: [requests, kv_heads, G, most, D] in 32 bits; positions
    [requests, most], and which rows there are."""
    q = s["q"].float()
    T, H, D = q.shape
    kv = s["k_pages"].shape[1]
    cu = s["cu_new"].long()
    t = torch.arange(s["max_new"], device=q.device)
    live = t < (cu[1:] - cu[:-1])[:, None]
    q = q[(cu[:-1, None] + t).clamp(max=T - 1)].unflatten(2, (kv, H // kv))
    return q.permute(0, 2, 3, 1, 4), s["context_lens"].long()[:, None] + t, live


def _by_token(s, x):
    """[requests, kv_heads, G, most, ..] -> [tokens, heads, ..]"""
    cu = s["cu_new"].long()
    i = torch.arange(s["q"].shape[0], device=x.device)
    r = torch.searchsorted(cu[1:], i, right=True)
    return x.permute(0, 3, 1, 2, *range(4, x.dim()))[r, i - cu[r]].flatten(1, 2)


def _seen(s, pos, key):
    """Whether a token at `pos` attends to position `key`."""
    return (key <= pos) & ((pos - key < (s["kernel"] or _FAR)) | (key < s["sinks"]))


def _cached(s, pages, table, key):
    """Rows at positions key [n, keys] of the tables' requests: [n, kv_heads, keys, D]."""
    page = s["page"]
    ids = table.gather(1, (key // page).clamp(max=table.shape[1] - 1)).clamp(min=0).long()
    return pages[ids, :, key % page].transpose(1, 2).float()


def _scores(s):
    """[requests, kv_heads, G, most, positions] in 32 bits, -inf where a token does not attend."""
    q, pos, live = _rows(s)
    R, kv, G, most, D = q.shape
    key = torch.arange(s["max_context"], device=q.device)
    k = _cached(s, s["k_pages"], s["page_table"], key.expand(R, -1))
    p = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(D))
    seen = _seen(s, pos[:, :, None], key) & live[:, :, None]
    return p.unflatten(2, (G, most)).masked_fill_(~seen[:, None, None], -math.inf)


def _plain_weights(s):
    """Every request padded to the longest context and the most new tokens."""
    q, _, live = _rows(s)
    R, kv, G, most, _ = q.shape
    cu = s["cu_new"].long()
    at = (cu[:-1, None] + torch.arange(most, device=q.device)).clamp(max=s["lse"].shape[0] - 1)
    lse = s["lse"][at].unflatten(2, (kv, G)).permute(0, 2, 3, 1)
    p = _scores(s).sub_(lse[..., None]).exp_()
    p = p.masked_fill_(~live[:, None, None, :, None], 0.0).sum((2, 3))
    if s["first"] is not None:
        p.masked_fill_(torch.arange(p.shape[-1], device=q.device) < s["first"][:, None, None], 0.0)
    s["weights"][:, :, :p.shape[-1]] += p
    return s["weights"]


def _plain_shared(s):
    """The shared keys against all rows of a group in one product, every request's own keys
    against its rows, one softmax over both."""
    q, pos, live = _rows(s)
    R, kv, G, most, D = q.shape
    dev, cu, shared = q.device, s["cu_groups"].long(), s["shared_lens"].long()
    groups, many, rows = shared.shape[0], s["requests_of_group"], G * most
    group = torch.searchsorted(cu[1:], torch.arange(R, device=dev), right=True)
    place = torch.arange(R, device=dev) - cu[group]
    member = (cu[:-1, None] + torch.arange(many, device=dev)).clamp(max=R - 1)
    n = shared[group][:, None]

    def to_groups(x):  # [R, kv, rows, ..] -> [groups, kv, many rows, ..]
        return x[member].transpose(1, 2).flatten(2, 3)

    def to_requests(x):  # and back
        return x.unflatten(2, (many, rows)).transpose(1, 2)[group, place]

    qr = q.flatten(2, 3)
    key = torch.arange(s["max_shared"], device=dev)
    table = s["page_table"][cu[:-1].clamp(max=R - 1)]
    mine = torch.arange(s["max_own"], device=dev) + n
    last = pos[:, :1] + live.sum(1, keepdim=True)

    def both(pages):  # the groups' shared rows, and each request's own; nothing behind them
        return (_cached(s, pages, table, key.expand(groups, -1)),
                _cached(s, pages, s["page_table"], mine)
                .masked_fill_((mine >= last)[:, None, :, None], 0.0))

    ks, ko = both(s["k_pages"])
    ps = to_requests(torch.matmul(to_groups(qr), ks.transpose(-1, -2).contiguous()))
    po = torch.matmul(qr, ko.transpose(-1, -2).contiguous())
    i, j = pos[:, :, None], key
    see = torch.cat([_seen(s, i, j) & (j < n[:, :, None]), _seen(s, i, mine[:, None])], -1)
    see &= live[:, :, None]
    p = torch.cat([ps, po], -1).mul_(1.0 / math.sqrt(D)).unflatten(2, (G, most))
    p.masked_fill_(~see[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1)
    vs, vo = both(s["v_pages"])
    p = p.flatten(2, 3)
    ps, po = p[..., :key.shape[0]].contiguous(), p[..., key.shape[0]:].contiguous()
    out = to_requests(torch.matmul(to_groups(ps), vs)) + torch.matmul(po, vo)
    out = out.unflatten(2, (G, most)) / total.clamp(min=1e-38)
    return _by_token(s, out).to(s["q"].dtype), _by_token(s, lse).contiguous()


def _plain_evict(s):
    """Sorted weights of every head, padded to the largest room."""
    w, page, budget = s["weights"], s["page"], s["budget"]
    R, kv, room = w.shape
    dev = w.device
    n = s["context_lens"].long()[:, None]
    first = torch.zeros_like(n) if s["first"] is None else s["first"].long()[:, None]
    first = first.clamp(0, budget)
    recent = torch.minimum(torch.full_like(first, s["recent"]), budget - first)
    over = n > budget
    j = torch.arange(room, device=dev)
    # the heaviest of those between the first and the last
    among = (over & (j >= first) & (j < n - recent))[:, None]
    keys = w.masked_fill(~among, -math.inf)
    order = torch.sort(keys, dim=-1, descending=True, stable=True).indices
    heavy = torch.zeros_like(w, dtype=torch.bool).scatter_(
        -1, order, (j < budget - first - recent)[:, None].expand_as(order)) & among
    # of each place the token that it gets: the last ones in order, of the others each its own
    # or, where that one goes, the next of the heavy ones behind the places
    end = (budget - recent)[:, None]
    hole = among & ~heavy & (j < end)
    behind = torch.sort(j.expand_as(w).masked_fill(~(heavy & (j >= end)), room), -1).values
    fill = behind.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0))
    kept = torch.where(hole, fill, j)
    kept = torch.where((over & (j >= budget - recent))[:, None], j + (n - budget)[:, None], kept)
    kept = kept[..., :budget]
    left = torch.minimum(n, torch.full_like(n, budget))
    took = j[:kept.shape[-1]] < left[:, :, None]
    at = kept.clamp(max=room - 1)
    weights = torch.zeros_like(w)
    weights[..., :kept.shape[-1]] = w.gather(-1, at).masked_fill_(~took, 0.0)
    table, heads = s["page_table"].long(), torch.arange(kv, device=dev)[None, :, None]
    to = j[:kept.shape[-1]].expand_as(kept)
    move = took & (kept != to)

    def spot(x):
        return table.gather(1, (x // page).flatten(1)).view_as(x)[move], \
            heads.expand_as(x)[move], (x % page)[move]

    src, dst = spot(at), spot(to)
    for pages in (s["k_pages"], s["v_pages"]):
        pages[dst] = pages[src]
    # freed pages: request by request behind the list's head
    col = torch.arange(table.shape[1], device=dev)
    freed = over & (col >= -(-budget // page)) & (col < (n + page - 1) // page)
    ids = table[freed].int()
    head = s["head"] - freed.sum().int()
    s["free_pages"][head.long() + torch.arange(ids.shape[0], device=dev)] = ids
    kept = kept.masked_fill(~took, -1).int()
    if kept.shape[-1] < budget:
        kept = torch.cat([kept, kept.new_full((R, kv, budget - kept.shape[-1]), -1)], -1)
    return left[:, 0].int(), weights, kept, head, s["free_pages"], s["k_pages"], s["v_pages"]


def run(s):
    if not own:
        return {"shared": _plain_shared, "weights": _plain_weights, "evict": _plain_evict}[
            s["op"]](s)
    import paper_2403_04690_amd as na

    if s["op"] == "shared":
        return na.cache_shared_attention(
            s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["context_lens"], s["cu_new"],
            s["cu_groups"], s["shared_lens"], s["kernel"] or None, s["sinks"],
            max_new=s["max_new"], max_shared=s["max_shared"], max_own=s["max_own"])
    if s["op"] == "weights":
        na.cache_weights(s["q"], s["lse"], s["k_pages"], s["page_table"], s["context_lens"],
                         s["cu_new"], s["weights"], s["kernel"] or None, s["sinks"],
                         first=s["first"], max_new=s["max_new"], max_context=s["max_context"])
        return s["weights"]
    return na.cache_evict(s["weights"], s["k_pages"], s["v_pages"], s["page_table"],
                          s["context_lens"], s["free_pages"], s["head"], s["budget"],
                          recent=s["recent"], first=s["first"]) \
        + (s["free_pages"], s["k_pages"], s["v_pages"])


# ---------------------------------------------------------------- 64 bits

def _weights64(q, k, i, j, kernel, sinks):
    """Logits of rows q at positions i over k at positions j in 64 bits, -inf where hidden."""
    dist = i[:, None] - j[None, :]
    hide = (dist < 0) | ((dist >= kernel) & (j[None, :] >= sinks))
    return (q @ k.T * q.shape[-1] ** -0.5).masked_fill_(hide, -math.inf)


def exact(case, seed):
    if case["op"] == "evict":
        return _exact_evict(case, seed)
    kernel, page, D = case["kernel"] or _FAR, case["page"], case["head_dim"]
    G, H = case["heads"] // case["kv_heads"], case["heads"]
    if case["op"] == "weights":
        ctx, new = _lens(case)
        s, first = _weights_inputs(case, seed), _first_lens(case)
        res = s["weights"].double()
    else:
        ctx, new, cu, shared = _lens(case)
        s = _shared_inputs(case, seed)
        out = torch.zeros(sum(new), H, D, dtype=torch.float64, device="cuda")
        res = torch.zeros(sum(new), H, dtype=torch.float64, device="cuda")
        group = [g for g in range(case["groups"]) for _ in range(cu[g], cu[g + 1])]
    table = s["page_table"].long()
    at = 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        j = torch.arange(c + n, device="cuda")
        ids = table[r][j // page]
        if case["op"] == "shared":
            g = group[r]
            ids[:shared[g]] = table[cu[g]][j[:shared[g]] // page]
        i = torch.arange(c, c + n, device="cuda").repeat_interleave(G)
        for h in range(case["kv_heads"]) if n else ():
            span = slice(h * G, (h + 1) * G)
            q = s["q"][at:at + n, span].double().reshape(n * G, D)
            a = _weights64(q, s["k_pages"][ids, h, j % page].double(), i, j, kernel,
                           case["sinks"])
            if case["op"] == "weights":
                lse = s["lse"][at:at + n, span].double().reshape(n * G, 1)
                w = a.sub_(lse).exp_().sum(0)
                res[r, h, first[r]:c + n] += w[first[r]:]
            else:
                lse = torch.logsumexp(a, -1)
                o = a.sub_(lse[:, None]).exp_() @ s["v_pages"][ids, h, j % page].double()
                out[at:at + n, span] = o.reshape(n, G, D)
                res[at:at + n, span] = lse.reshape(n, G)
        at += n
    return res if case["op"] == "weights" else (out, res)


def _exact_evict(case, seed):
    """Rows and weights where they belong; whole numbers have no value in 64 bits."""
    s = _evict_inputs(case, seed)
    ctx, first = _evict_lens(case)
    budget, page = case["budget"], case["page"]
    w, table = s["weights"].cpu(), s["page_table"].cpu().long()
    weights = torch.zeros_like(w).double()
    k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
    for r, n in enumerate(ctx):
        for h in range(case["kv_heads"]):
            if n <= budget:
                weights[r, h, :n] = w[r, h, :n].double()
                continue
            f = min(first[r], budget)
            last = min(case["recent"], budget - f)
            # (a stable ascending sort of the negated values: of equal ones the first)
            more = (-w[r, h, f:n - last]).numpy().argsort(kind="stable")[:budget - f - last] + f
            heavy, end = set(more.tolist()), budget - last
            behind = iter(sorted(x for x in heavy if x >= end))
            keep = torch.tensor([i if i < f or i in heavy else next(behind) for i in range(end)]
                                + [*range(n - last, n)], dtype=torch.int64)
            weights[r, h, :budget] = w[r, h, keep].double()
            to = torch.arange(budget)
            src = (table[r, keep // page].cuda(), h, (keep % page).cuda())
            dst = (table[r, to // page].cuda(), h, (to % page).cuda())
            for pages, given in ((k_pages, s["k_pages"]), (v_pages, s["v_pages"])):
                pages[dst] = given[src].double()
    return None, weights.cuda(), None, None, None, k_pages, v_pages
