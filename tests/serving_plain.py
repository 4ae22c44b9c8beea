"""Plain 64-bit forms of the cache operators for long contexts, and how far a kernel may be from
them (see sequence_plain.py for the bounds of scores, exponentials and sums).

Parts.  A row's result is joined from parts of its keys in fp32: each part's logsumexp is off by
U |lse| from its rounding and by an exponential's and a logarithm's error, 2^-21 each, and weighs
the part with another exponential.  All of it is relative to a part's weight, so the joined mean
moves by at most twice that (numerator and sum) times (P |V|), and the mean of each part is rounded to
fp32 once more.

Weights.  exp(s - lse) is off by the score's error, by U (|s| + 2 |lse|) from the difference and from
the conversion of the logsumexp to base 2, and by exp2's 2^-21, all relative; n of them are summed in
fp32 (n U of the sum), and added to what was there (U of the result).
"""
import math

import torch

from tests import sequence_plain as plain

U = plain.U


def groups_of(requests, cu_groups, shared):
    """(first request, shared tokens) of each request; (itself, 0) outside of all groups."""
    res = [(r, 0) for r in range(requests)]
    for g, n in enumerate(shared):
        for r in range(max(cu_groups[g], 0), min(cu_groups[g + 1], requests)):
            res[r] = (max(cu_groups[g], 0), max(n, 0))
    return res


def places(page_table, of, r, tokens, page):
    """(page, row) of positions 0 .. tokens - 1 of request r; page -1 where there is none."""
    first, shared = of[r]
    res = []
    for j in range(tokens):
        ids = page_table[first if j < shared else r]
        res.append((ids[j // page] if j // page < len(ids) else -1, j % page))
    return res


def rows_at(pages, places):
    """[Hkv, len(places), D] in float64; zeros where the page does not exist."""
    P = pages.shape[0]
    ids = torch.tensor([a if 0 <= a < P else 0 for a, _ in places], dtype=torch.int64)
    at = torch.tensor([b for _, b in places], dtype=torch.int64)
    ok = torch.tensor([0 <= a < P for a, _ in places], dtype=torch.bool)
    rows = pages[ids, :, at].double() if P else torch.zeros((len(places),) + (
        pages.shape[1], pages.shape[3])).double()
    return torch.where(ok[:, None, None], rows, torch.zeros(1).double()).transpose(0, 1)


def shared(q, k_pages, v_pages, page_table, context, new, cu_groups, shared_lens, kernel_size,
           sinks, scale):
    """New tokens [T, H, D] over the cache: out, lse, tolerances."""
    dtype, G, page = q.dtype, q.shape[1] // k_pages.shape[1], k_pages.shape[2]
    q, k_pages, v_pages = (t.detach().cpu() for t in (q, k_pages, v_pages))
    of = groups_of(len(context), cu_groups, shared_lens)
    T, H, D = q.shape
    out, tol = torch.zeros(T, H, D).double(), torch.zeros(T, H, D).double()
    lse, tol_lse = torch.zeros(T, H).double(), torch.zeros(T, H).double()
    at = 0
    for r, (c, n) in enumerate(zip(context, new)):
        j = torch.arange(c + n)
        seen = plain.visible(torch.arange(c, c + n), j, kernel_size, sinks)
        keep = seen.any(0)[None, :, None]  # (what no token sees may be anything)
        where = places(page_table, of, r, c + n, page)
        ks, vs = (torch.where(keep, rows_at(x, where), torch.zeros(1).double())
                  for x in (k_pages, v_pages))
        for h in range(H):
            o, e, t, te = plain.attend(q[at:at + n, h].double(), ks[h // G], vs[h // G], seen,
                                       scale, dtype)
            s = (q[at:at + n, h].double() @ ks[h // G].T) * scale
            p = torch.where(seen, torch.exp(s - e[:, None]), torch.zeros_like(s))
            far = torch.where(seen, s.abs(), torch.zeros_like(s)).amax(-1) if n else e
            e_p = U * (far + e.abs()) + 2 * 2.0 ** -21
            out[at:at + n, h], lse[at:at + n, h] = o, e
            tol[at:at + n, h] = t + (2 * e_p + U)[:, None] * (p @ vs[h // G].abs())
            tol_lse[at:at + n, h] = te + 2 * e_p
        at += n
    return out, lse, tol, tol_lse


def weights(q, lse, k_pages, page_table, context, new, before, kernel_size, sinks, scale,
            first=None):
    """What the weights become, and the tolerance."""
    G, page = q.shape[1] // k_pages.shape[1], k_pages.shape[2]
    q, lse, k_pages = (t.detach().cpu() for t in (q, lse, k_pages))
    res = before.detach().cpu().double()
    tol = torch.zeros_like(res)
    H, D, capacity = q.shape[1], q.shape[2], res.shape[2]
    of = [(r, 0) for r in range(len(context))]
    at = 0
    for r, (c, n) in enumerate(zip(context, new)):
        j = torch.arange(c + n)
        seen = plain.visible(torch.arange(c, c + n), j, kernel_size, sinks)
        keep = seen.any(0)[None, :, None]
        ks = torch.where(keep, rows_at(k_pages, places(page_table, of, r, c + n, page)),
                         torch.zeros(1).double())
        f = 0 if first is None else max(first[r], 0)
        got = (seen.any(0) & (j >= f))[:capacity]
        m = got.shape[0]
        for h in range(H):
            qq, e = q[at:at + n, h].double(), lse[at:at + n, h, None].double()
            s = (qq @ ks[h // G].T) * scale
            p = torch.where(seen, torch.exp(s - e), torch.zeros_like(s))
            off = (D + 4) * U * abs(scale) * (qq.abs() @ ks[h // G].abs().T) \
                + 2 * U * (s.abs() + 2 * e.abs()) + 2.0 ** -21 + (G * n + 2) * U
            res[r, h // G, :m] += torch.where(got, p.sum(0)[:m], torch.zeros(m).double())
            tol[r, h // G, :m] += torch.where(got, (p * off).sum(0)[:m], torch.zeros(m).double())
        tol[r, :, :m] += 2 * U * res[r, :, :m].abs() * got
        at += n
    return res, tol


def evict(weights, k_pages, v_pages, page_table, context, free, head, budget, recent=0, first=None):
    """(context, weights, kept, head, free list, k_pages, v_pages) after an eviction, token by
    token."""
    R, Hkv, capacity = weights.shape
    P, page = k_pages.shape[0], k_pages.shape[2]
    w = weights.detach().cpu()
    k_pages, v_pages = (t.detach().cpu() for t in (k_pages, v_pages))
    new_k, new_v = k_pages.clone(), v_pages.clone()
    new_w, kept = torch.zeros_like(w), torch.full((R, Hkv, budget), -1, dtype=torch.int32)
    free, back, after = list(free), [], []
    for r in range(R):
        n = min(max(context[r], 0), len(page_table[r]) * page)
        f = 0 if first is None else min(max(first[r], 0), budget)
        last = min(recent, budget - f)
        end = budget - last
        after.append(min(n, budget))
        for c in range(Hkv):
            at = list(range(n))
            if n > budget:
                def rank(i):
                    x = float(w[r, c, i]) if i < capacity else 0.0
                    return (1, 0.0, i) if math.isnan(x) else (0, -x, i)

                heavy = set(sorted(range(f, n - last), key=rank)[:budget - f - last])
                behind = iter(sorted(i for i in heavy if i >= end))
                at = [i if i < f or i in heavy else next(behind) for i in range(end)]
                assert next(behind, None) is None
                at += range(n - last, n)
            for i, j in enumerate(at):
                kept[r, c, i] = j
                if i < capacity:
                    new_w[r, c, i] = w[r, c, j] if j < capacity else 0.0
                to, src = page_table[r][i // page], page_table[r][j // page]
                if n > budget and i != j and 0 <= to < P:
                    for a, b in ((new_k, k_pages), (new_v, v_pages)):
                        a[to, c, i % page] = b[src, c, j % page] if 0 <= src < P else 0
        if n > budget:
            back += [x for x in page_table[r][-(-budget // page):-(-n // page)] if 0 <= x < P]
    base = head - len(back)
    for i, x in enumerate(back):
        if 0 <= base + i < len(free):
            free[base + i] = x
    return after, new_w, kept, max(base, 0), free, new_k, new_v
