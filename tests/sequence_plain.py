"""Plain 64-bit forms of the sequence operators, and how far a kernel may be from them.

Bounds.  A kernel works from the same (already rounded) inputs.  u is half a step of the type
(relative), U = 2^-24 that of fp32.
  * a score is a sum of D products in fp32, then two more roundings (times scale, minus the
    reference): off by e_s <= (D + 4) U scale sum_c |q_c k_c|, and by U times the distance from
    the reference (|s| + |lse|), both relative errors of exp(s) with it;
  * exp2 in hardware and the sums of P (n terms in any order): at most 2^-21 + n U together,
    n U as a worst case is far above what is seen, 32 U covers the tree of partial sums and
    the joins;
  * P is rounded to the type: u relative, and 2^-25 absolute in fp16 below its normal range
    (against the row's largest P, which is at least 1);
  * out is a P-weighted mean, so each relative error of P moves it by at most that times
    (P |V|), once from the numerator and once from the sum, and it is rounded once more.

Gradients start from the logsumexp that the forward stored, like the kernels: P = exp(s - lse).
  * dout . v is a sum of D products in fp32: off by (D + 2) U of its absolute sum;
  * delta is sum_j P_j dout . v_j.  A kernel sums that (off by P's relative error of each term
    and by P times the error of dout . v), or takes dout . out of the stored out, a sum of D
    products too: off by (D + 2) U of its absolute sum, and by dout . (out - sum_j P_j v_j),
    which is known;
  * dA = P (dout . v - delta) is off by the relative errors of P (its score's, exp2's) and by P
    times those sums' errors, then rounded to the type (u, and 2^-25 absolute in fp16);
  * dq, dk and dv sum n such terms in fp32, at most n U of their absolute sum more, and are
    rounded once.
"""
import math

import torch

U = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.float16, torch.bfloat16)}


def visible(i, j, kernel_size, sinks):
    """[len(i), len(j)]: whether position i attends to position j."""
    d = i[:, None] - j[None, :]
    return (d >= 0) & ((d < kernel_size) | (j[None, :] < sinks))


def attend(q, k, v, seen, scale, dtype):
    """out, logsumexp of rows q [n, D] over k, v [m, D] (float64), and their bounds."""
    s = (q @ k.T) * scale
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1) if k.shape[0] else torch.full((q.shape[0],), -math.inf).double()
    p = torch.where(seen, torch.exp(s - lse[:, None]), torch.zeros_like(s))
    out = p @ v
    size = abs(scale) * (q.abs() @ k.abs().T)
    far = torch.where(seen, s.abs() + lse.abs()[:, None], torch.zeros_like(s))
    e_s = torch.where(seen, (q.shape[1] + 4) * U * size + 2 * U * far, torch.zeros_like(s))
    e_s = e_s.amax(-1) if k.shape[0] else torch.zeros(q.shape[0]).double()
    e_p = 2.0 ** -21 + 32 * U
    u = HALF[dtype]
    mean = p @ v.abs()
    u_p = u if dtype != torch.float32 else 0.0
    tol = (u_p + 2 * (e_s + e_p))[:, None] * mean + u * out.abs() + 1e-30
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25 * (seen.double() @ v.abs()) + 2.0 ** -25
    tol_lse = e_s + e_p + 4 * U * (1 + torch.where(lse.isfinite(), lse.abs(), 0 * lse))
    return out, lse, tol, tol_lse


def sink(q, k, v, kernel_size, sinks, scale, lengths=None):
    """[B, H, N, D] over [B, Hkv, N, D]: out, lse, tolerances (float64 on the CPU)."""
    dtype = q.dtype
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    B, H, N, D = q.shape
    G = H // k.shape[1]
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float64)
    tol_lse = torch.zeros_like(lse)
    for b in range(B):
        n = N if lengths is None else max(0, min(N, int(lengths[b])))
        pos = torch.arange(n)
        seen = visible(pos, pos, kernel_size, sinks)
        for h in range(H):
            c = h // G
            r = attend(q[b, h, :n], k[b, c, :n], v[b, c, :n], seen, scale, dtype)
            out[b, h, :n], lse[b, h, :n], tol[b, h, :n], tol_lse[b, h, :n] = r
    return out, lse, tol, tol_lse


def sink_grad(q, k, v, out, lse, dout, kernel_size, sinks, scale, lengths=None):
    """dq, dk, dv and their tolerances (float64 on the CPU) from the stored out and lse."""
    dtype = q.dtype
    q, k, v, out, lse, dout = (t.detach().cpu().double() for t in (q, k, v, out, lse, dout))
    B, H, N, D = q.shape
    G = H // k.shape[1]
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    tols = [torch.zeros_like(t) for t in (q, k, v)]
    u = HALF[dtype]
    u_p = u if dtype != torch.float32 else 0.0
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    for b in range(B):
        n = N if lengths is None else max(0, min(N, int(lengths[b])))
        pos = torch.arange(n)
        seen = visible(pos, pos, kernel_size, sinks)
        for h in range(H):
            c = h // G
            qq, kk, vv = q[b, h, :n], k[b, c, :n], v[b, c, :n]
            g, o = dout[b, h, :n], out[b, h, :n]
            s = (qq @ kk.T) * scale
            p = torch.where(seen, torch.exp(s - lse[b, h, :n, None]), torch.zeros_like(s))
            e = (D + 4) * U * abs(scale) * (qq.abs() @ kk.abs().T) \
                + 2 * U * (s.abs() + lse[b, h, :n, None].abs()) + 2.0 ** -21
            dp, size = g @ vv.T, g.abs() @ vv.abs().T
            da = p * (dp - (p * dp).sum(-1, keepdim=True))
            e_delta = (p * (e * dp.abs() + (D + 2) * U * size)).sum(-1, keepdim=True) \
                + (g * (o - p @ vv)).sum(-1, keepdim=True).abs() \
                + (D + 2) * U * (g * o).abs().sum(-1, keepdim=True)
            e_da = (e + u_p) * da.abs() + tiny * seen + (1 + e) * p * (
                (D + 2) * U * size + e_delta)
            e_p = p * (e + u_p) + tiny * seen
            grads[0][b, h, :n] = scale * da @ kk
            tols[0][b, h, :n] = abs(scale) * (e_da + n * U * da.abs()) @ kk.abs()
            grads[1][b, c, :n] += scale * da.T @ qq
            tols[1][b, c, :n] += abs(scale) * (e_da + G * n * U * da.abs()).T @ qq.abs()
            grads[2][b, c, :n] += p.T @ g
            tols[2][b, c, :n] += (e_p + G * n * U * p).T @ g.abs()
    return grads, [t + u * g.abs() + tiny for t, g in zip(tols, grads)]


def tables(context, new, page_table, free, page_size, tokens, head=0):
    """The tables of a step, token by token; page_table is a nested list, updated."""
    cu, slots, positions = [0], [-1] * tokens, [-1] * tokens
    taken, at = head, 0
    for r, (c, n) in enumerate(zip(context, new)):
        c, n = max(c, 0), max(n, 0)
        row, most = page_table[r], len(page_table[r])
        fresh = {}
        for x in range(-(-c // page_size), min(-(-(c + n) // page_size), most)):
            fresh[x] = free[taken] if 0 <= taken < len(free) else -1
            taken += 1
        for t in range(n):
            x = (c + t) // page_size
            page = -1
            if x < most:
                page = fresh[x] if x in fresh else row[x]
            if at < tokens:
                positions[at] = c + t
                slots[at] = -1 if page < 0 else page * page_size + (c + t) % page_size
                if x in fresh and (c + t) % page_size == 0:
                    row[x] = page
            at += 1
        cu.append(at)
    return cu, slots, positions, taken


def cached(pages, ids, tokens):
    """Rows of one request: pages [P, Hkv, page, D] by its ids (float64); [Hkv, tokens, D]."""
    P, Hkv, page, D = pages.shape
    rows = torch.zeros(Hkv, tokens, D, dtype=torch.float64)
    for x in range(-(-tokens // page)):
        n = min(page, tokens - x * page)
        if x < len(ids) and 0 <= ids[x] < P:
            rows[:, x * page:x * page + n] = pages[ids[x], :, :n].double()
    return rows


def cache(q, k_pages, v_pages, page_table, context, new, kernel_size, sinks, scale):
    """New tokens [T, H, D] over the cache: out, lse, tolerances."""
    dtype, G = q.dtype, q.shape[1] // k_pages.shape[1]
    q, k_pages, v_pages = (t.detach().cpu() for t in (q, k_pages, v_pages))
    T, H, D = q.shape
    out, tol = torch.zeros(T, H, D).double(), torch.zeros(T, H, D).double()
    lse, tol_lse = torch.zeros(T, H).double(), torch.zeros(T, H).double()
    at = 0
    for r, (c, n) in enumerate(zip(context, new)):
        pos = torch.arange(c, c + n)
        j = torch.arange(c + n)
        seen = visible(pos, j, kernel_size, sinks)
        # (what no token sees may be anything)
        keep = seen.any(0)[None, :, None]
        ks, vs = (torch.where(keep, cached(x, page_table[r], c + n), torch.zeros(1).double())
                  for x in (k_pages, v_pages))
        for h in range(H):
            res = attend(q[at:at + n, h].double(), ks[h // G], vs[h // G], seen, scale, dtype)
            out[at:at + n, h], lse[at:at + n, h], tol[at:at + n, h], tol_lse[at:at + n, h] = res
        at += n
    return out, lse, tol, tol_lse


def close(got, want, tol, what):
    got = got.detach().cpu().double()
    both = (got == want) | ((got - want).abs() <= tol)
    if not bool(both.all()):
        off = ((got - want).abs() / tol.clamp(min=1e-300))[~both]
        raise AssertionError(f"{what}: {int((~both).sum())} of {both.numel()} outside, worst "
                             f"{float(off.nan_to_num(math.inf).max()):.3g} tolerances")
