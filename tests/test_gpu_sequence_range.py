"""fp16 over its whole range: weights far below 1, output gradients that are small or large, and rows
of very different size.  A weight is rounded once, relative to itself, wherever it lies.

Bounds are those of tests/sequence_plain.py without its allowance for fp16's subnormal numbers in
each pair.  What stays of them:
  * P enters dv times 2^15: 2^-25 of that, 2^-40 absolute;
  * dA is scaled so that the largest of a row (for dq) or of a key (for dk) is at least 2^11: 2^-36
    of that largest one;
  * a stored gradient is rounded to fp16: 2^-25 absolute below its normal range.
"""
import math

import pytest
import torch

from tests import sequence_plain as plain

pytestmark = pytest.mark.gpu

U, HALF = plain.U, plain.HALF[torch.float16]


@pytest.fixture(scope="module")
def na():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    import paper_2403_04690_amd as lib

    lib.load_library()
    return lib


def _normal(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _grads(q, k, v, out, lse, g, W, S):
    """dq, dk, dv of one sequence and their bounds (float64 on the CPU)."""
    q, k, v, out, lse, g = (t.detach().cpu().double()[0] for t in (q, k, v, out, lse, g))
    H, N, D = q.shape
    G, scale = H // k.shape[0], D ** -0.5
    seen = plain.visible(torch.arange(N), torch.arange(N), W, S)
    want = [torch.zeros_like(t) for t in (q, k, v)]
    tol = [torch.zeros_like(t) for t in (q, k, v)]
    for h in range(H):
        c = h // G
        s = scale * q[h] @ k[c].T
        p = torch.where(seen, torch.exp(s - lse[h, :, None]), torch.zeros_like(s))
        e = (D + 4) * U * scale * (q[h].abs() @ k[c].abs().T) \
            + 2 * U * (s.abs() + lse[h, :, None].abs()) + 2.0 ** -21
        dp, size = g[h] @ v[c].T, g[h].abs() @ v[c].abs().T
        da = p * (dp - (p * dp).sum(-1, keepdim=True))
        e_delta = (p * (e * dp.abs() + (D + 2) * U * size)).sum(-1, keepdim=True) \
            + (g[h] * (out[h] - p @ v[c])).sum(-1, keepdim=True).abs() \
            + (D + 2) * U * (g[h] * out[h]).abs().sum(-1, keepdim=True)
        e_da = (e + HALF) * da.abs() + (1 + e) * p * ((D + 2) * U * size + e_delta)
        e_row = (e_da + 2.0 ** -36 * da.abs().amax(1, keepdim=True)) * seen
        e_key = (e_da + 2.0 ** -36 * da.abs().amax(0, keepdim=True)) * seen
        want[0][h] = scale * da @ k[c]
        tol[0][h] = scale * (e_row + N * U * da.abs()) @ k[c].abs()
        want[1][c] += scale * da.T @ q[h]
        tol[1][c] += scale * (e_key + G * N * U * da.abs()).T @ q[h].abs()
        want[2][c] += p.T @ g[h]
        tol[2][c] += (p * (e + HALF) + 2.0 ** -40 * seen + G * N * U * p).T @ g[h].abs()
    return want, [t + HALF * w.abs() + 2.0 ** -25 for t, w in zip(tol, want)]


SHAPES = [
    # heads, kv_heads, tokens, head_dim, kernel_size, sinks
    (2, 2, 512, 64, 512, 0),
    (4, 2, 300, 128, 300, 0),
    (1, 1, 400, 32, 90, 0),
    (6, 2, 700, 64, 40, 5),      # first tokens' rows in workgroups of their own, heads split
    (8, 2, 500, 128, 64, 40),
    (3, 1, 260, 32, 33, 4),
]


def _check(na, q, k, v, g, W, S):
    q, k, v, g = (t.half().cuda() for t in (q, k, v, g))
    out, lse = na.sink_forward(q, k, v, W, S)
    got = na.sink_backward(q, k, v, out, lse, g, W, S)
    want, tol = _grads(q, k, v, out, lse, g, W, S)
    for name, a, w, t in zip(("dq", "dk", "dv"), got, want, tol):
        assert bool((w.abs() < 6e4).all())  # (the gradient itself is inside fp16)
        plain.close(a[0], w, t, name)


@pytest.mark.parametrize("H,Hkv,N,D,W,S", SHAPES)
def test_small_output_gradients_keep_their_digits(na, H, Hkv, N, D, W, S):
    """dout of 2^-14: dA lies where fp16 has few digits or none; large keys and queries bring dq and
    dk back."""
    q, k, v, g = (_normal((1, h, N, D), i) for i, h in enumerate((H, Hkv, Hkv, H)))
    _check(na, q / 16, 16 * k, v, g * 2.0 ** -14, W, S)   # (scores as of q and k)
    _check(na, 16 * q, k / 16, v, g * 2.0 ** -14, W, S)


@pytest.mark.parametrize("H,Hkv,N,D,W,S", SHAPES)
def test_large_output_gradients_stay_finite(na, H, Hkv, N, D, W, S):
    """P (dout . v - delta) beyond fp16's largest number, with gradients inside it."""
    q, k, v, g = (_normal((1, h, N, D), 10 + i) for i, h in enumerate((H, Hkv, Hkv, H)))
    _check(na, q / 4, k / 4, 32 * v, g * 2.0 ** 10, W, S)


@pytest.mark.parametrize("order", ["growing", "shrinking", "mixed", "zeros"])
@pytest.mark.parametrize("H,Hkv,N,D,W,S", SHAPES)
def test_rows_of_very_different_size(na, H, Hkv, N, D, W, S, order):
    """Output gradients from 2^-14 to 2^9 in one sequence, in any order, and rows of zeros."""
    q, k, v, g = (_normal((1, h, N, D), 20 + i) for i, h in enumerate((H, Hkv, Hkv, H)))
    at = torch.arange(N) / (N - 1)
    if order == "mixed":
        at = at[torch.randperm(N, generator=torch.Generator().manual_seed(1))]
    elif order == "shrinking":
        at = 1 - at
    size = 2.0 ** (23 * at - 14)
    if order == "zeros":
        size = torch.where(torch.arange(N) % 70 < 40, 0.0, size)
    _check(na, q, k, v, g * size[:, None], W, S)


def _rms(x):
    return float(x.double().pow(2).mean().sqrt())


def test_gradients_over_a_long_context(na):
    """Weights of 2^-17.  Roundings are independent: their squares add up, u / sqrt(3) of a value at
    most each (uniform over a step; 4096 values show it within 1.1 %, 1.1 allows for that and for
    the products' fp32 sums), beside exp2's 2^-21, taken at its worst."""
    N, D = 2 ** 17 - 5, 64
    gen = torch.Generator("cuda").manual_seed(3)
    q, k, v, g = (torch.randn(1, 1, N, D, generator=gen, device="cuda", dtype=torch.float16)
                  for _ in range(4))
    out, lse = na.sink_forward(q, k, v, N)
    dq, dk, dv = na.sink_backward(q, k, v, out, lse, g, N)
    qd, kd, vd, gd, od = (t[0, 0].double() for t in (q, k, v, g, out))
    scale, ld = D ** -0.5, lse[0, 0].double()
    delta = (gd * od).sum(-1)
    keys = torch.randperm(N // 2, generator=torch.Generator().manual_seed(4))[:64].cuda() + N // 4
    s = scale * qd @ kd[keys].T
    seen = keys[None, :] <= torch.arange(N, device="cuda")[:, None]
    p = torch.where(seen, torch.exp(s - ld[:, None]), torch.zeros_like(s))
    da = p * (gd @ vd[keys].T - delta[:, None])
    rows = torch.randperm(N // 2, generator=torch.Generator().manual_seed(5))[:64].cuda() + N // 2
    sr = scale * qd[rows] @ kd.T
    pr = torch.where(torch.arange(N, device="cuda")[None, :] <= rows[:, None],
                     torch.exp(sr - ld[rows, None]), torch.zeros_like(sr))
    dr = pr * (gd[rows] @ vd.T - delta[rows, None])
    for name, got, a, b in (("dv", dv[0, 0, keys], p.T, gd), ("dk", dk[0, 0, keys], scale * da.T, qd),
                            ("dq", dq[0, 0, rows], scale * dr, kd)):
        want = a @ b
        each = HALF / math.sqrt(3) * ((a ** 2 @ b ** 2) + want ** 2).sqrt()
        bound = 1.1 * _rms(each) + 2.0 ** -21 * _rms(a.abs() @ b.abs())
        # (values are stored in fp16: 2^-25 at most below its normal range)
        bound += 2.0 ** -25 / math.sqrt(3)
        assert _rms(got.double() - want) < bound, (name, _rms(got.double() - want) / bound)


@pytest.mark.parametrize("form", ["sequence", "cache"])
def test_forward_beside_a_key_that_takes_most_of_the_weight(na, form):
    """A first token with score 12 above the others and little in its value (as sinks come out of
    training): the others' weights are e^-12 of it, and are what the output is made of.  Errors
    as above: P and out are rounded once."""
    N, D = 2 ** 16 - 5, 64
    gen = torch.Generator().manual_seed(6)
    q, k, v = (torch.randn(1, 1, N, D, generator=gen) for _ in range(3))
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[0, 0, 0] = 0.0
    k[0, 0, 0, 0] = 12.0                     # 8 * 12 / sqrt(64)
    v[0, 0, 0] = 0.0
    q, k, v = (t.half().cuda() for t in (q, k, v))
    rows = torch.arange(N - 64, N, device="cuda")
    if form == "sequence":
        out = na.sink_forward(q, k, v, N)[0][0, 0, rows]
    else:
        pages = -(-N // 16)
        kp, vp = (torch.nn.functional.pad(t[0, 0], (0, 0, 0, 16 * pages - N)).reshape(pages, 1, 16, D)
                  for t in (k, v))
        table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        out = na.cache_attention(q[0, 0, rows][:, None].contiguous(), kp, vp, table, ints(N - 64),
                                 ints(0, 64))[0][:, 0]
        one = na.cache_attention(q[0, 0, rows[-1:]][:, None].contiguous(), kp, vp, table, ints(N - 1),
                                 ints(0, 1), max_new=1)[0][:, 0]
        out = torch.cat([out, one])
        rows = torch.cat([rows, rows[-1:]])
    s = D ** -0.5 * q[0, 0, rows].double() @ k[0, 0].double().T
    s = s.masked_fill(torch.arange(N, device="cuda")[None, :] > rows[:, None], -math.inf)
    p = torch.softmax(s, -1)
    want = p @ v[0, 0].double()
    each = HALF / math.sqrt(3) * ((p ** 2 @ v[0, 0].double() ** 2) + want ** 2).sqrt()
    bound = 1.1 * _rms(each) + 2.0 ** -20 * _rms(p @ v[0, 0].double().abs()) + 2.0 ** -25
    assert _rms(out.double() - want) < bound, _rms(out.double() - want) / bound


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hkv,N,D,W,S", SHAPES)
def test_an_overflowed_output_gradient_shows(na, dtype, H, Hkv, N, D, W, S):
    """An infinite dout (a loss scale that was too high) makes every gradient that it reaches
    infinite or NaN, so that a training program can skip the step, and none of another key head's.
    (Keys of its own that the row does not see may be hit too: their P is 0, and 0 times infinity
    is NaN in the plain form as well.)"""
    q, k, v, g = (_normal((1, h, N, D), 30 + i).to(dtype).cuda()
                  for i, h in enumerate((H, Hkv, Hkv, H)))
    out, lse = na.sink_forward(q, k, v, W, S)
    want = na.sink_backward(q, k, v, out, lse, g, W, S)
    row, head = 2 * N // 3, H - 1
    g = g.clone()
    g[0, head, row, 7] = math.inf
    got = na.sink_backward(q, k, v, out, lse, g, W, S)
    seen = plain.visible(torch.tensor([row]), torch.arange(N), W, S)[0].cuda()
    hit = [torch.zeros(t.shape[:3], dtype=torch.bool, device="cuda") for t in want]
    hit[0][0, head, row] = True
    hit[1][0, Hkv - 1, seen] = True
    hit[2][0, Hkv - 1, seen] = True
    for name, a, w, h in zip(("dq", "dk", "dv"), got, want, hit):
        # (dv takes dout itself: only its column; dq and dk its product with every value)
        bad = ~a[..., 7].isfinite() if name == "dv" else (~a.isfinite()).all(-1)
        assert bool(bad[h].all()), name
        others = slice(0, head) if name == "dq" else slice(0, Hkv - 1)
        assert torch.equal(a[:, others], w[:, others]), name
