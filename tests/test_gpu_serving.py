"""The cache operators for long contexts on the GPU against their plain 64-bit forms."""
import functools
import math
import random

import pytest
import torch

from tests import sequence_plain as plain
from tests import serving_plain as ref

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
WHOLE = 2 ** 31 - 1


@pytest.fixture(scope="module")
def na():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_04690_amd as lib

    lib.load_library()
    return lib


def _randn(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(DT[dtype])


def _int(x):
    return torch.tensor(x, dtype=torch.int32).reshape(-1).cuda()


def _offsets(new):
    return _int([sum(new[:i]) for i in range(len(new) + 1)])


def _tables(context, new, page, cu_groups, shared, seed=0, spare=3, most=None):
    """Page table (nested list) in a random order over a pool, its size, and the pages left over.
    Whole shared pages are the group's first request's."""
    of = ref.groups_of(len(context), cu_groups, shared)
    need = [-(-(c + n) // page) for c, n in zip(context, new)]
    own = [w - min(w, s // page if f != r else 0) for r, (w, (f, s)) in enumerate(zip(need, of))]
    order = list(range(sum(own) + spare))
    random.Random(seed).shuffle(order)
    most = max(need + [1]) if most is None else most
    table = []
    for r, (f, s) in enumerate(of):
        row = list(table[f][:need[r] - own[r]]) if f != r else []
        row += [order.pop() for _ in range(own[r])]
        table.append((row + [-1] * most)[:max(most, len(row))])
    return table, len(order) + sum(own), order


def _poison(pages, places):
    """NaN in every row that is not one of places."""
    keep = torch.zeros(pages.shape[0], pages.shape[2], dtype=torch.bool)
    for a, b in places:
        if 0 <= a < keep.shape[0]:
            keep[a, b] = True
    pages.masked_fill_(~keep.to(pages.device)[:, None, :, None], math.nan)


def _seen_places(table, of, context, new, page, W, S):
    res = set()
    for r, (c, n) in enumerate(zip(context, new)):
        seen = plain.visible(torch.arange(c, c + n), torch.arange(c + n), W, S).any(0)
        res |= {p for p, s in zip(ref.places(table, of, r, c + n, page), seen.tolist()) if s}
    return res


# ---------------------------------------------------------------- shared first tokens

def _shared_check(na, own, new, cu_groups, shared, H, Hkv, D, page, dtype, W=None, S=0, seed=0,
                  scale=None, table=None, **hints):
    """own: cached tokens of each request behind its group's shared ones."""
    of = ref.groups_of(len(own), cu_groups, shared)
    context = [max(0, c + s) for c, (_, s) in zip(own, of)]
    made, P, _ = _tables(context, new, page, cu_groups, shared, seed)
    table = made if table is None else table
    kp, vp = (_randn((P, Hkv, page, D), dtype, seed + 1 + i) for i in range(2))
    q = _randn((sum(new), H, D), dtype, seed + 3)
    w = WHOLE if W is None else W
    s = 1 / math.sqrt(D) if scale is None else scale
    want = ref.shared(q, kp, vp, table, context, new, cu_groups, shared, w, S, s)
    for t in (kp, vp):
        _poison(t, _seen_places(table, of, context, new, page, w, S))
    out, lse = na.cache_shared_attention(
        q, kp, vp, torch.tensor(table, dtype=torch.int32).cuda(), _int(context), _offsets(new),
        _int(cu_groups), _int(shared), W, S, scale, **hints)
    torch.cuda.synchronize()
    plain.close(out, want[0], want[2], "out")
    plain.close(lse, want[1], want[3], "lse")
    return out, lse


SHARED_CASES = [
    # own, new, cu_groups, shared, heads, kv_heads, head_dim, page, dtype, kernel_size, sinks
    ([0], [1], [0, 1], [0], 1, 1, 32, 16, "fp32", None, 0),
    ([0], [1], [0, 1], [1], 1, 1, 32, 16, "fp16", None, 0),
    ([0, 0], [1, 1], [0, 2], [40], 4, 2, 64, 16, "bf16", None, 0),
    ([5, 70, 0], [1, 1, 1], [0, 3], [300], 2, 2, 32, 16, "fp32", None, 0),
    ([5, 70, 0, 33], [1] * 4, [0, 4], [515], 16, 4, 128, 64, "bf16", None, 0),
    ([5, 70, 0, 33], [1] * 4, [0, 4], [515], 8, 8, 64, 32, "fp16", None, 0),
    # groups of none, one and several requests; requests before and behind all groups
    ([9, 40, 3, 20, 0, 31], [1, 2, 1, 0, 3, 1], [1, 1, 2, 5], [50, 77, 129], 6, 2, 64, 16, "fp16",
     None, 0),
    ([9, 40, 3, 20, 0, 31], [1, 2, 1, 0, 3, 1], [1, 1, 2, 5], [50, 77, 129], 6, 2, 128, 16, "fp32",
     None, 0),
    # windows: inside the own tokens, into the shared ones, and with first tokens of both
    ([50, 90], [1, 3], [0, 2], [200], 4, 1, 64, 16, "bf16", 20, 0),
    ([50, 90], [1, 3], [0, 2], [200], 4, 1, 64, 16, "fp16", 100, 4),
    ([5, 40, 200], [2, 1, 30], [0, 3], [70], 4, 4, 32, 16, "fp32", 33, 90),
    ([5, 40, 200], [2, 1, 30], [0, 3], [70], 4, 2, 128, 16, "bf16", 1, 1),
    ([20, 9], [3, 1], [0, 2], [70], 200, 2, 32, 16, "fp16", 60, 2),
    # a whole block of heads of one token, and more
    ([3, 3], [1, 1], [0, 2], [100], 64, 1, 64, 16, "bf16", None, 0),
    # chunks of prompts
    ([0, 0, 7], [60, 130, 1], [0, 3], [150], 4, 2, 64, 16, "bf16", None, 0),
    ([0, 20], [200, 90], [0, 2], [333], 3, 3, 128, 32, "fp16", None, 0),
    ([0, 20], [70, 50], [0, 2], [333], 6, 1, 32, 16, "fp32", 64, 3),
]


@pytest.mark.parametrize("own,new,cu,shared,H,Hkv,D,page,dtype,W,S", SHARED_CASES)
def test_shared_attention(na, own, new, cu, shared, H, Hkv, D, page, dtype, W, S):
    # without hints; with exact ones; and with hints that are wrong
    exact = {"max_new": max(new), "max_shared": max(shared),
             "max_own": max(c + n for c, n in zip(own, new))}
    for hints in ({}, exact, {"max_new": 1, "max_shared": 1, "max_own": 1},
                  {"max_new": 5000, "max_shared": 2 ** 30, "max_own": 2 ** 30}):
        _shared_check(na, own, new, cu, shared, H, Hkv, D, page, dtype, W, S, **hints)


@pytest.mark.parametrize("dtype,D", [("fp16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 32)])
@pytest.mark.parametrize("new", [[1, 1, 1], [90, 1, 4]])
def test_long_shared_tokens_are_split_and_joined(na, dtype, D, new):
    own, hint = [900, 0, 31], {"max_new": max(new), "max_shared": 4000, "max_own": 1000}
    _shared_check(na, own, new, [0, 3], [4000], 4, 2, D, 16, dtype, **hint)
    _shared_check(na, own, new, [0, 1, 3], [700, 3333], 4, 2, D, 64, dtype, 3000, 5, **hint)
    # one workgroup for all shared keys of its rows, and for all own ones
    few = {"max_new": max(new), "max_shared": 1, "max_own": 1}
    _shared_check(na, own, new, [0, 3], [4000], 4, 2, D, 16, dtype, **few)
    _shared_check(na, [3000, 2500, 5], new, [0, 2, 3], [700, 90], 4, 2, D, 32, dtype, 2300, 70, **few)


def test_shared_tokens_reach_past_a_context(na):
    """Tokens that are new to a request but shared by its group are read on the group's pages."""
    _shared_check(na, [-60, -10, 5], [30, 1, 2], [0, 3], [100], 4, 2, 64, 16, "fp16")
    _shared_check(na, [-100, 3], [3, 40], [0, 2], [100], 4, 2, 32, 16, "fp32", 20, 2)


@pytest.mark.parametrize("groups", [1, 70])
def test_more_requests_and_groups_than_a_wave(na, groups):
    R = 150
    rng = random.Random(groups)
    cu = [0] + sorted(rng.randint(0, R) for _ in range(groups - 1)) + [R]
    shared = [rng.randint(0, 60) for _ in range(groups)]
    new = [rng.choice((0, 1, 1, 2)) for _ in range(R)]
    own = [rng.randint(0, 40) for _ in range(R)]
    for W, S in ((None, 0), (30, 3)):
        _shared_check(na, own, new, cu, shared, 4, 2, 32, 16, "fp32", W, S, max_new=2)
    _shared_check(na, own, [70] + new[1:], cu, shared, 4, 2, 64, 16, "bf16")


def test_one_pages_table_or_another_makes_no_difference(na):
    """With a table that lists the shared pages for everybody, cache_attention agrees."""
    context, new, page, H, Hkv, D = [300, 260, 257], [1, 1, 3], 16, 8, 2, 64
    table, P, _ = _tables(context, new, page, [0, 3], [256])
    kp, vp = (_randn((P, Hkv, page, D), "fp32", i) for i in range(2))
    q = _randn((5, H, D), "fp32", 2)
    t = torch.tensor(table, dtype=torch.int32).cuda()
    a = na.cache_attention(q, kp, vp, t, _int(context), _offsets(new))
    b = na.cache_shared_attention(q, kp, vp, t, _int(context), _offsets(new), _int([0, 3]),
                                  _int([256]))
    want = ref.shared(q, kp, vp, table, context, new, [0, 3], [256], WHOLE, 0, D ** -0.5)
    for x, y, w, tol in zip(a, b, want[:2], want[2:]):
        plain.close(x, w, tol, "cache_attention")
        plain.close(y, w, tol, "cache_shared_attention")


def test_no_groups_at_all(na):
    _shared_check(na, [100, 3], [1, 2], [0], [], 4, 2, 64, 16, "bf16")
    _shared_check(na, [100, 3], [60, 2], [0], [], 4, 2, 64, 16, "bf16")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_shared_attention_of_strided_tensors(na, dtype):
    own, new, cu, shared, H, Hkv, D, page = [5, 70], [2, 1], [0, 2], [90], 4, 2, 64, 16
    context = [95, 160]
    table, P, _ = _tables(context, new, page, cu, shared)
    kp, vp = (_randn((P, Hkv, page, D), dtype, i) for i in range(2))
    q = _randn((H, 3, 2 * D), dtype, 5)[:, :, D:].transpose(0, 1)  # [tokens, heads, D]
    out = torch.full((3, 2 * H, D + 16), 7.0, dtype=DT[dtype], device="cuda")[:, ::2, :D]
    want = ref.shared(q, kp, vp, table, context, new, cu, shared, WHOLE, 0, D ** -0.5)
    args = (torch.tensor(table, dtype=torch.int32).cuda(), _int(context), _offsets(new), _int(cu),
            _int(shared))
    got, lse = na.cache_shared_attention(q, kp, vp, *args, out=out)
    assert got is out
    plain.close(out, want[0], want[2], "out")
    base = out._base if out._base is not None else out
    assert bool((base[:, 1::2] == 7.0).all()) and bool((base[:, :, D:] == 7.0).all())
    # one query row for all heads: a stride of 0
    q0 = _randn((3, 1, D), dtype, 6).expand(3, H, D)
    want = ref.shared(q0, kp, vp, table, context, new, cu, shared, WHOLE, 0, D ** -0.5)
    plain.close(na.cache_shared_attention(q0, kp, vp, *args)[0], want[0], want[2], "out")


def test_shared_attention_leaves_rows_behind_the_last_token(na):
    table, P, _ = _tables([40, 50], [1, 2], 16, [0, 2], [33])
    kp, vp = (_randn((P, 2, 16, 64), "bf16", i) for i in range(2))
    q = _randn((9, 4, 64), "bf16", 3)
    for hint in ({}, {"max_new": 2}):
        out = torch.full((9, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((9, 4), 5.0, device="cuda")
        na.cache_shared_attention(q, kp, vp, torch.tensor(table).int().cuda(), _int([40, 50]),
                                  _int([0, 1, 3]), _int([0, 2]), _int([33]), out=out, lse=lse,
                                  **hint)
        assert bool((out[3:] == 5).all()) and bool((lse[3:] == 5).all())
        assert not bool((lse[:3] == 5).any())


@pytest.mark.parametrize("new", [[1, 1], [50, 3]])
def test_shared_pages_that_do_not_exist_are_zeros(na, new):
    own, cu, shared = [30, 10], [0, 2], [100]
    context = [130, 110]
    made, P, _ = _tables(context, new, 16, cu, shared)
    table = [list(row) for row in made]
    table[0][2], table[0][4], table[1][6], table[1][0] = -1, P, 2 ** 31 - 1, -2 ** 31
    _shared_check(na, own, new, cu, shared, 4, 2, 64, 16, "fp16", table=table)


def test_offsets_and_groups_that_make_no_sense_stay_inside(na):
    """Decreasing and far offsets: which rows are written is open, memory is not."""
    R, T, H, Hkv, D, page = 6, 12, 4, 2, 64, 16
    kp, vp = (_randn((9, Hkv, page, D), "bf16", i) for i in range(2))
    table = torch.randint(0, 9, (R, 4), dtype=torch.int32).cuda()
    q = _randn((T, H, D), "bf16", 3)
    big = 2 ** 31 - 1
    for cu in ([0, 5, 3, 12, 2, 8, 12], [0, 2, 4, 6, 8, 10, big], [-5, 2, 4, 1, big, -big, 12]):
        for groups, shared in (([0, 3, 6], [20, 30]), ([4, 1, 6], [big, 10]),
                               ([-7, big, 2, 9], [5, -3, 40]), ([2, 2, 2, 2], [9, 9, 9])):
            for hint in ({}, {"max_new": 1}):
                out, lse = na.cache_shared_attention(
                    q, kp, vp, table, _int([10, 70, big, -3, 50, 0]), _int(cu), _int(groups),
                    _int(shared), **hint)
                torch.cuda.synchronize()
    assert out.shape == q.shape


def test_shared_attention_repeats_bit_for_bit(na):
    runs = [_shared_check(na, [5, 70, 0, 33], [3, 1, 9, 1], [0, 2, 4], [515, 90], 8, 2, 64, 16,
                          "bf16", max_new=9) for _ in range(3)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


def test_shared_attention_of_nothing(na):
    kp = torch.zeros(3, 2, 16, 32, dtype=torch.float16, device="cuda")
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    for T, H in ((0, 4), (5, 0)):
        k = kp if H else kp[:, :0]
        out, lse = na.cache_shared_attention(
            torch.zeros(T, H, 32, dtype=torch.float16, device="cuda"), k, k, table, _int([3, 3]),
            _int([0, 0, T]), _int([0, 2]), _int([3]))
        assert out.shape == (T, H, 32) and lse.shape == (T, H)
    # an empty pool and an empty table read as zeros
    out, lse = na.cache_shared_attention(
        _randn((2, 4, 32), "fp16", 1), kp[:0], kp[:0], table[:, :0], _int([3, 3]), _int([0, 1, 2]),
        _int([0, 2]), _int([3]))
    assert bool((out == 0).all())


def test_pages_beyond_32_bit_offsets(na):
    """A pool of more than 2^32 bytes, whose last pages are the shared ones."""
    Hkv, page, D, P = 8, 128, 128, 17000
    kp = torch.zeros(P, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    assert kp.numel() * 2 > 2 ** 32
    ids = [P - 1, 3, P - 2]
    for t, seed in ((kp, 1), (vp, 2)):
        for i in ids:
            t[i] = _randn((Hkv, page, D), "bf16", seed * 100 + i % 97)
    q = _randn((2, 16, D), "bf16", 4)
    small = [t[ids] for t in (kp, vp)]
    want = ref.shared(q, *small, [[0, 1], [0, 2]], [200, 150], [1, 1], [0, 2], [100], WHOLE, 0,
                      D ** -0.5)
    out, lse = na.cache_shared_attention(
        q, kp, vp, torch.tensor([[ids[0], ids[1]], [ids[0], ids[2]]]).int().cuda(),
        _int([200, 150]), _int([0, 1, 2]), _int([0, 2]), _int([100]), max_new=1)
    plain.close(out, want[0], want[2], "out")
    weights = torch.zeros(2, Hkv, 300, device="cuda")
    na.cache_weights(q, lse, kp, torch.tensor([[ids[0], ids[1]], [ids[0], ids[2]]]).int().cuda(),
                     _int([200, 150]), _int([0, 1, 2]), weights, max_new=1)
    want, tol = ref.weights(q, lse, small[0], [[0, 1], [0, 2]], [200, 150], [1, 1],
                            torch.zeros(2, Hkv, 300), WHOLE, 0, D ** -0.5)
    plain.close(weights, want, tol, "weights")
    # and the rows there move
    w = torch.rand(2, Hkv, 256, device="cuda")
    table = [[ids[1], ids[0]], [ids[2], 0]]
    small = [torch.stack([t[ids[1]], t[ids[0]], t[ids[2]]]) for t in (kp, vp)]
    want = ref.evict(w, *small, [[0, 1], [2, -1]], [200, 90], [0] * 5, 5, 100, 10)
    got = na.cache_evict(w, kp, vp, torch.tensor(table).int().cuda(), _int([200, 90]),
                         _int([0] * 5), _int([5]), 100, 10)
    assert torch.equal(got[2].cpu(), want[2])
    for t, x in ((kp, want[5]), (vp, want[6])):
        assert torch.equal(torch.stack([t[ids[1]], t[ids[0]], t[ids[2]]]).cpu(), x)


# ---------------------------------------------------------------- gathered weights

def _weights_check(na, context, new, H, Hkv, D, page, dtype, W=None, S=0, first=None, seed=0,
                   capacity=None, scale=None, table=None, **hints):
    made, P, _ = _tables(context, new, page, [0], [], seed)
    table = made if table is None else table
    kp, vp = (_randn((P, Hkv, page, D), dtype, seed + 1 + i) for i in range(2))
    q = _randn((sum(new), H, D), dtype, seed + 3)
    w = WHOLE if W is None else W
    s = 1 / math.sqrt(D) if scale is None else scale
    lse = ref.shared(q, kp, vp, table, context, new, [0], [], w, S, s)[1].float().cuda()
    of = ref.groups_of(len(context), [0], [])
    want_k = kp.clone()
    _poison(kp, _seen_places(table, of, context, new, page, w, S))
    room = len(table[0]) * page if capacity is None else capacity
    gen = torch.Generator(device="cuda").manual_seed(seed + 9)
    weights = torch.rand((len(context), Hkv, room), generator=gen, device="cuda") * 0.01
    before = weights.clone()
    want, tol = ref.weights(q, lse, want_k, table, context, new, before, w, S, s, first)
    na.cache_weights(q, lse, kp, torch.tensor(table, dtype=torch.int32).cuda(), _int(context),
                     _offsets(new), weights, W, S, scale,
                     first=None if first is None else _int(first), **hints)
    torch.cuda.synchronize()
    plain.close(weights, want, tol, "weights")
    assert torch.equal(weights.cpu()[tol == 0], before.cpu()[tol == 0])
    return weights


WEIGHT_CASES = [
    # context, new, heads, kv_heads, head_dim, page, dtype, kernel_size, sinks, first
    ([0], [1], 1, 1, 32, 16, "fp32", None, 0, None),
    ([40], [1], 4, 1, 64, 16, "fp16", None, 0, None),
    ([5, 700, 31, 32, 64], [1] * 5, 8, 2, 128, 16, "bf16", None, 0, None),
    ([5, 700, 31, 32, 64], [1, 1, 0, 1, 1], 16, 4, 64, 32, "fp16", 100, 4, [0, 2, 9, 100, 33]),
    ([1000, 900], [1, 1], 8, 8, 128, 64, "fp32", 33, 40, None),
    ([0, 0, 50], [1, 0, 2], 4, 4, 32, 16, "bf16", 1, 0, [-3, 0, 2 ** 31 - 1]),
    ([300], [1], 64, 1, 64, 16, "bf16", None, 0, None),     # a group of two blocks of rows
    ([300, 20], [7, 9], 12, 2, 32, 16, "fp32", None, 0, None),
    ([0], [200], 4, 2, 64, 16, "bf16", None, 0, None),      # a prompt
    ([77, 0, 500], [130, 1, 63], 6, 2, 64, 16, "fp16", None, 0, [10, 0, 333]),
    ([77, 0, 500], [130, 1, 63], 6, 2, 128, 64, "bf16", 50, 20, None),
    ([77, 0, 500, 9], [130, 0, 63, 0], 5, 1, 32, 128, "fp32", 50, 3, None),
    ([600], [300], 3, 3, 128, 16, "fp32", None, 0, None),
    ([600], [300], 3, 3, 64, 16, "fp32", 7, 0, None),
    ([2000], [40], 2, 2, 32, 16, "fp16", 300, 16, [5]),
    ([900, 0], [33, 257], 14, 2, 128, 16, "bf16", 700, 1, None),
    ([200, 3], [9, 3], 200, 2, 32, 16, "fp16", 60, 2, None),  # heads of a token over several stages
    ([200, 3], [9, 30], 48, 1, 64, 16, "bf16", None, 0, None),
]


@pytest.mark.parametrize("context,new,H,Hkv,D,page,dtype,W,S,first", WEIGHT_CASES)
def test_weights(na, context, new, H, Hkv, D, page, dtype, W, S, first):
    most, longest = max(new), max(c + n for c, n in zip(context, new))
    for hints in ({}, {"max_new": most, "max_context": longest},
                  {"max_new": 1, "max_context": 1}, {"max_new": 5000, "max_context": 2 ** 30}):
        _weights_check(na, context, new, H, Hkv, D, page, dtype, W, S, first, **hints)


@pytest.mark.parametrize("capacity", [0, 1, 33, 100, 1000])
def test_weights_behind_the_capacity_are_not_kept(na, capacity):
    for new in ([1, 1], [50, 3]):
        _weights_check(na, [90, 40], new, 4, 2, 64, 16, "fp16", capacity=capacity, first=[3, 0])


@pytest.mark.parametrize("dtype,D", [("fp16", 128), ("fp32", 32)])
def test_weights_of_long_contexts(na, dtype, D):
    _weights_check(na, [9000, 1290], [1, 1], 4, 2, D, 16, dtype, max_new=1, max_context=9001)
    _weights_check(na, [5000, 1290], [1, 90], 4, 2, D, 64, dtype, 4000, 4, max_new=90)
    # one workgroup for all keys of a request
    _weights_check(na, [5000, 1290], [1, 1], 4, 2, D, 16, dtype, max_new=1, max_context=1)
    _weights_check(na, [2500, 700], [1, 90], 4, 2, D, 16, dtype, max_new=90, max_context=1)


def test_weights_of_many_requests(na):
    R = 90
    rng = random.Random(2)
    _weights_check(na, [rng.randint(0, 70) for _ in range(R)],
                   [rng.choice((0, 1, 1, 3)) for _ in range(R)], 4, 2, 32, 16, "bf16")


@pytest.mark.parametrize("new", [[1, 1], [50, 3]])
def test_weights_of_pages_that_do_not_exist_are_those_of_zero_keys(na, new):
    made, P, _ = _tables([130, 110], new, 16, [0], [])
    table = [list(row) for row in made]
    table[0][2], table[0][4], table[1][3], table[1][0] = -1, P, 2 ** 31 - 1, -2 ** 31
    _weights_check(na, [130, 110], new, 4, 2, 64, 16, "fp16", table=table)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
def test_weights_scales(na, scale):
    _weights_check(na, [60], [5], 4, 2, 32, 16, "fp32", scale=scale)
    _weights_check(na, [60], [50], 4, 2, 32, 16, "fp32", scale=scale)


def test_weights_of_a_row_sum_to_its_new_tokens(na):
    """Every new token gives a weight of 1 a query head."""
    context, new, H, Hkv = [700, 90], [3, 120], 8, 2
    table, P, _ = _tables(context, new, 16, [0], [])
    kp, vp = (_randn((P, Hkv, 16, 64), "fp32", i) for i in range(2))
    q = _randn((sum(new), H, 64), "fp32", 3)
    t, c, cu = torch.tensor(table).int().cuda(), _int(context), _offsets(new)
    _, lse = na.cache_attention(q, kp, vp, t, c, cu, 300, 4)
    weights = torch.zeros(2, Hkv, 800, device="cuda")
    na.cache_weights(q, lse, kp, t, c, cu, weights, 300, 4)
    n = torch.tensor(new).double()[:, None] * H / Hkv
    assert bool(((weights.cpu().double().sum(-1) - n).abs() <= n * 2.0 ** -16).all())


def test_weights_of_the_last_tokens_of_a_chunk(na):
    """A slice of the rows, with the lengths that belong to it."""
    H, Hkv, D = 4, 2, 64
    table, P, _ = _tables([100], [60], 16, [0], [])
    kp, vp = (_randn((P, Hkv, 16, D), "bf16", i) for i in range(2))
    q = _randn((60, H, D), "bf16", 3)
    t = torch.tensor(table).int().cuda()
    _, lse = na.cache_attention(q, kp, vp, t, _int([100]), _int([0, 60]))
    weights = torch.zeros(1, Hkv, 160, device="cuda")
    na.cache_weights(q[-7:], lse[-7:], kp, t, _int([153]), _int([0, 7]), weights)
    want, tol = ref.weights(q[-7:], lse[-7:], kp, table, [153], [7], torch.zeros(1, Hkv, 160),
                            WHOLE, 0, D ** -0.5)
    plain.close(weights, want, tol, "weights")


def test_weights_of_offsets_that_make_no_sense_stay_inside(na):
    R, T, H, Hkv, D = 6, 12, 4, 2, 64
    kp = _randn((9, Hkv, 16, D), "bf16", 1)
    table = torch.randint(0, 9, (R, 4), dtype=torch.int32).cuda()
    q, lse = _randn((T, H, D), "bf16", 3), torch.zeros(T, H, device="cuda")
    big = 2 ** 31 - 1
    for cu in ([0, 5, 3, 12, 2, 8, 12], [0, 2, 4, 6, 8, 10, big], [-5, 2, 4, 1, big, -big, 12]):
        for hint in ({}, {"max_new": 1}):
            weights = torch.zeros(R, Hkv, 70, device="cuda")
            na.cache_weights(q, lse, kp, table, _int([10, 70, big, -3, 50, 0]), _int(cu), weights,
                             **hint)
            torch.cuda.synchronize()


def test_weights_repeat_bit_for_bit(na):
    for new in ([3, 1], [60, 100]):
        a, b = (_weights_check(na, [300, 77], new, 6, 2, 64, 16, "fp16") for _ in range(2))
        assert torch.equal(a, b)


# ---------------------------------------------------------------- eviction

def _evict_check(na, w, context, D, page, dtype, budget, recent=0, first=None, seed=0, table=None,
                 spare=3, most=None, head=None, free=None):
    R, Hkv, _ = w.shape
    made, P, order = _tables([max(c, 0) for c in context], [0] * R, page, [0], [], seed,
                             spare=spare, most=most)
    table = made if table is None else table
    kp, vp = (_randn((P, Hkv, page, D), dtype, seed + 1 + i) for i in range(2))
    used = sum(-(-max(c, 0) // page) for c in context)
    # a list of all pages, those of the requests in front of its head
    free = [-7] * used + order if free is None else free
    head = used if head is None else head
    want = ref.evict(w, kp, vp, table, context, free, head, budget, recent, first)
    gfree = _int(free)
    ctx, gtable = _int(context), torch.tensor(table, dtype=torch.int32).reshape(R, -1).cuda()
    wdev, h = w.cuda(), _int([head])
    got = na.cache_evict(wdev, kp, vp, gtable, ctx, gfree, h, budget, recent,
                         None if first is None else _int(first))
    torch.cuda.synchronize()
    assert got[0].tolist() == want[0]
    assert torch.equal(got[2].cpu(), want[2])
    # (NaN equal to NaN)
    assert torch.equal(got[1].cpu().view(torch.int32), want[1].view(torch.int32))
    assert got[3].tolist() == [want[3]]
    assert gfree.tolist() == want[4]
    assert torch.equal(kp.cpu(), want[5]) and torch.equal(vp.cpu(), want[6])
    # what is read stays
    assert torch.equal(wdev.cpu().view(torch.int32), w.view(torch.int32)) and ctx.tolist() == context
    assert gtable.tolist() == [list(r) for r in table] and h.tolist() == [head]
    return got


def _weights(R, Hkv, capacity, seed=0, ties=False):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn((R, Hkv, capacity), generator=gen).mul(3).exp()
    if ties:
        w = w.log2().round().exp2()  # a few values, many times each
    return w * (torch.rand((R, Hkv, capacity), generator=gen) > 0.1)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("context,Hkv,D,page,dtype,budget,recent,first", [
    ([1], 1, 32, 16, "fp32", 1, 0, None),
    ([2], 1, 32, 16, "fp16", 1, 0, None),
    ([2], 1, 32, 16, "fp16", 1, 1, None),
    ([17, 0, 16], 2, 64, 16, "bf16", 16, 0, None),
    ([100, 30, 64], 2, 64, 16, "bf16", 40, 8, None),
    ([100, 30, 64], 3, 128, 32, "fp32", 40, 0, [4, 4, 50]),
    ([100, 90, 64], 1, 128, 16, "fp16", 50, 50, None),      # the last ones alone
    ([100, 90, 64], 1, 64, 16, "fp16", 50, 20, [30, 50, 2 ** 31 - 1]),
    ([100, 90, 64], 1, 64, 16, "fp16", 50, 0, [-5, 49, 50]),
    ([100, 90, 64], 1, 64, 16, "fp16", 50, 2 ** 40, [1, 0, 49]),
    ([51, 90, 64], 2, 32, 128, "bf16", 50, 10, [0, 3, 0]),  # one too many
    ([700, 1030, 999, 5], 2, 64, 64, "bf16", 333, 45, [16] * 4),
])
def test_evict(na, context, Hkv, D, page, dtype, budget, recent, first, ties):
    w = _weights(len(context), Hkv, max(context) + 7, ties=ties)
    _evict_check(na, w, context, D, page, dtype, budget, recent, first)


@pytest.mark.parametrize("n,budget,recent", [
    (9000, 100, 10), (9000, 8500, 600), (5000, 4097, 4000), (4096, 4095, 0), (12289, 4096, 4096),
    (30000, 1, 0), (32768, 20000, 0), (40000, 5000, 100), (33001, 33000, 1), (70001, 40000, 7)])
def test_evict_of_long_contexts(na, n, budget, recent):
    _evict_check(na, _weights(2, 1, n, ties=n % 2 == 0), [n, n - 1], 32, 64, "fp16", budget, recent,
                 [3, 0])


def test_evict_of_equal_weights_keeps_the_first(na):
    for value, n in ((v, n) for v in (0.0, 1.0, -2.5, math.inf, -math.inf, math.nan) for n in (9000, 36000)):
        w = torch.full((1, 1, n), value)
        got = _evict_check(na, w, [n], 32, 64, "fp32", 5000, 7)
        assert got[2][0, 0].tolist() == list(range(4993)) + list(range(n - 7, n))


def test_evict_of_weights_that_are_no_numbers(na):
    """NaN of both signs is below everything, infinities and zeros of both signs are in their
    places, and weights that differ in their last digit are told apart."""
    gen = torch.Generator().manual_seed(3)
    odd = torch.tensor([math.nan, -math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45,
                        torch.finfo(torch.float32).max, -torch.finfo(torch.float32).max, 1.0,
                        1.0 + 2.0 ** -23, 1.0 - 2.0 ** -24, -1.0, -1.0 - 2.0 ** -23])
    for n, budget in ((40, 20), (300, 100), (300, 290), (5000, 2500), (40000, 11111)):
        w = odd[torch.randint(0, odd.numel(), (2, 2, n), generator=gen)]
        _evict_check(na, w, [n, n - 3], 32, 16, "fp32", budget, 3)


@pytest.mark.parametrize("capacity", [0, 1, 40, 64, 99])
def test_evict_weights_behind_the_capacity_are_0(na, capacity):
    _evict_check(na, _weights(2, 2, capacity), [100, 80], 64, 16, "bf16", 50, 5)
    _evict_check(na, -_weights(2, 2, capacity), [100, 80], 64, 16, "bf16", 50, 5)


def test_evict_of_many_requests(na):
    rng = random.Random(4)
    R = 150
    context = [rng.choice((0, -4, rng.randint(1, 90))) for _ in range(R)]
    first = [rng.randint(-1, 40) for _ in range(R)]
    _evict_check(na, _weights(R, 2, 90), context, 32, 16, "fp16", 30, 6, first)


def test_evict_returns_pages_of_very_many_requests(na):
    """More requests, and more freed pages, than are looked at in one go."""
    rng = random.Random(7)
    R = 2100
    context = [rng.choice((0, 5, rng.randint(1, 80))) for _ in range(R)]
    _evict_check(na, _weights(R, 1, 80), context, 32, 16, "fp16", 17, 3)
    _evict_check(na, _weights(2, 1, 40000), [40000, 39000], 32, 16, "fp16", 5000, 3)
    table, P, _ = _tables([40000, 39000], [0, 0], 16, [0], [])
    for r, x in ((0, 400), (0, 1999), (1, 2000), (1, 313)):
        table[r][x] = -1
    _evict_check(na, _weights(2, 1, 40000), [40000, 39000], 32, 16, "fp16", 5000, 3, table=table)


def test_evict_pages_that_do_not_exist(na):
    w = _weights(2, 2, 200)
    table, P, _ = _tables([200, 150], [0, 0], 16, [0], [])
    table[0][1], table[0][9], table[1][3], table[1][8], table[0][11] = -1, P, 2 ** 31 - 1, -5, -9
    _evict_check(na, w, [200, 150], 64, 16, "fp16", 60, 9, table=table)


def test_evict_clamps_lengths_to_the_table(na):
    _evict_check(na, _weights(2, 2, 200), [100, 64], 64, 16, "fp16", 60, 9,
                 table=[[3, 1, 4, 0, 5], [9, 2, 6, 8, 7]])


def test_evict_returns_what_the_list_has_room_for(na):
    w = _weights(2, 1, 200)
    for head, size in ((0, 4), (3, 4), (9, 4), (12, 30), (2, 0), (2 ** 31 - 1, 5), (-2 ** 31, 5)):
        _evict_check(na, w, [200, 150], 32, 16, "fp32", 60, 9, head=head, free=[-3] * size)


def test_evict_leaves_shared_first_tokens(na):
    """Requests that share the pages of their first tokens keep them as they are."""
    table = [[0, 1, 2, 3, 4], [0, 1, 5, 6, 7], [0, 1, 8, 9, 10]]
    kp, vp = (_randn((11, 2, 16, 64), "bf16", i) for i in range(2))
    shared = kp[:2].clone(), vp[:2].clone()
    w = _weights(3, 2, 80)
    want = ref.evict(w, kp, vp, table, [80, 70, 75], [0] * 9, 9, 50, 5, [32] * 3)
    got = na.cache_evict(w.cuda(), kp, vp, torch.tensor(table).int().cuda(), _int([80, 70, 75]),
                         _int([0] * 9), _int([9]), 50, 5, _int([32] * 3))
    assert torch.equal(kp.cpu(), want[5]) and torch.equal(vp.cpu(), want[6])
    assert torch.equal(kp[:2], shared[0]) and torch.equal(vp[:2], shared[1])
    assert torch.equal(got[2].cpu(), want[2])


def test_evict_of_nothing(na):
    kp = torch.zeros(3, 2, 16, 32, dtype=torch.float16, device="cuda")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    got = na.cache_evict(torch.zeros(0, 2, 10, device="cuda"), kp, kp.clone(),
                         none.reshape(0, 4), none, _int([1, 2]), _int([1]), 5)
    assert got[0].numel() == 0 and got[2].shape == (0, 2, 5) and got[3].tolist() == [1]
    # a pool without pages
    got = na.cache_evict(_weights(1, 2, 40).cuda(), kp[:0], kp[:0].clone(),
                         torch.full((1, 4), -1, dtype=torch.int32).cuda(), _int([40]), _int([1, 2]),
                         _int([1]), 5)
    assert got[0].tolist() == [5] and got[3].tolist() == [1]


def test_evict_repeats_bit_for_bit(na):
    w = _weights(3, 2, 700, ties=True)
    runs = [_evict_check(na, w, [700, 600, 3], 64, 16, "bf16", 300, 30) for _ in range(3)]
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


# ---------------------------------------------------------------- together

class _Model:
    """The cache of one request in float64: its tokens of every head, in the order of places."""

    def __init__(self, Hkv):
        self.k, self.v, self.w = ([[] for _ in range(Hkv)] for _ in range(3))

    def add(self, k, v):
        for c in range(len(self.k)):
            self.k[c] += list(k[:, c])
            self.v[c] += list(v[:, c])
            self.w[c] += [0.0] * k.shape[0]


def _serve(na, dtype, steps, budget, recent, prompt=37, every=3, H=4, Hkv=2, D=64, page=16,
           capture=False):
    """Requests behind one prompt, served step by step with evictions in between; each step is
    checked against a model that holds every head's tokens as lists."""
    R = len(steps[0])
    most, P = 12, 12 * R + 4
    kp, vp = (torch.full((P, Hkv, page, D), math.nan, dtype=DT[dtype], device="cuda")
              for _ in range(2))
    pool = torch.randperm(P, generator=torch.Generator().manual_seed(1)).int().cuda()
    table = torch.full((R, most), -1, dtype=torch.int32, device="cuda")
    head = _int([0])
    scale, G = D ** -0.5, H // Hkv
    # the prompt, written once by request 0; its whole pages are everybody's, and each request has
    # the page in which it ends for itself
    pk, pv = (_randn((prompt, Hkv, D), dtype, 5 + i) for i in range(2))
    t = na.cache_tables(_int([0] * R), _int([prompt] + [0] * (R - 1)), table, pool, page, prompt,
                        head=head)
    na.cache_write(pk, pv, t[1], kp, vp)
    head = t[3]
    whole = prompt // page
    table[1:, :whole] = table[0, :whole]
    if prompt % page:
        table[1:, whole] = pool[head.item():head.item() + R - 1]
        for r in range(1, R):
            for pages in (kp, vp):
                pages[table[r, whole].long()] = pages[table[0, whole].long()]
        head = head + R - 1
    models = [_Model(Hkv) for _ in range(R)]
    for m in models:
        m.add(pk.double().cpu(), pv.double().cpu())
    ctx = _int([prompt] * R)
    first, groups, shared = _int([prompt] * R), _int([0, R]), _int([prompt])
    weights = torch.zeros(R, Hkv, most * page, device="cuda")
    evicted = 0
    for turn, new in enumerate(steps):
        T = sum(new)
        q, k, v = (_randn((T, h, D), dtype, 100 + 3 * turn + i) for i, h in enumerate((H, Hkv, Hkv)))
        lens = _int(new)
        cu, slots, _, head = na.cache_tables(ctx, lens, table, pool, page, T, head=head)
        na.cache_write(k, v, slots, kp, vp)
        out, lse = na.cache_shared_attention(q, kp, vp, table, ctx, cu, groups, shared)
        na.cache_weights(q, lse, kp, table, ctx, cu, weights, first=first)
        ctx = ctx + lens
        at, old = 0, weights.cpu()
        for r, n in enumerate(new):
            m = models[r]
            had = len(m.k[0])
            m.add(k[at:at + n].double().cpu(), v[at:at + n].double().cpu())
            seen = plain.visible(torch.arange(had, had + n), torch.arange(had + n), WHOLE, 0)
            for h in range(H):
                c = h // G
                ks, vs = torch.stack(m.k[c]), torch.stack(m.v[c])
                want = plain.attend(q[at:at + n, h].double().cpu(), ks, vs, seen, scale, DT[dtype])
                plain.close(out[at:at + n, h], want[0], 1.5 * want[2], f"turn {turn} out")
                plain.close(lse[at:at + n, h], want[1], 1.5 * want[3] + 2.0 ** -20, "lse")
                p = torch.where(seen, torch.exp((q[at:at + n, h].double().cpu() @ ks.T) * scale
                                                - want[1][:, None]), 0.0).sum(0)
                for j in range(prompt, had + n):
                    m.w[c][j] += float(p[j])
            for c in range(Hkv):
                w = torch.tensor(m.w[c])
                assert float((old[r, c, :had + n] - w).abs().max()) < 1e-4
            at += n
        if turn % every == every - 1:
            given = weights.clone()
            ctx, weights, kept, head = na.cache_evict(given, kp, vp, table, ctx, pool, head, budget,
                                                      recent, first)
            for r, m in enumerate(models):
                n = min(len(m.k[0]), budget)
                evicted += len(m.k[0]) - n
                for c in range(Hkv):
                    ids = kept[r, c, :n].tolist()
                    assert ids[:prompt] == list(range(prompt)) and len(set(ids)) == n
                    if len(m.k[0]) > budget:
                        # nothing that went was heavier than what stayed
                        gone = set(range(len(m.k[0]))) - set(ids)
                        stay = set(ids) - set(range(prompt)) - set(ids[n - recent:])
                        w = given[r, c].tolist()
                        assert max(w[i] for i in gone) <= min(w[i] for i in stay)
                    m.k[c] = [m.k[c][i] for i in ids]
                    m.v[c] = [m.v[c][i] for i in ids]
                    m.w[c] = [m.w[c][i] for i in ids]
            assert ctx.tolist() == [len(m.k[0]) for m in models]
    assert evicted > 0
    # no page is listed twice: what requests hold of their own and what is free
    mine = [int(x) for r in range(R) for x in table[r, whole:-(-int(ctx[r]) // page)]]
    rest = mine + [int(x) for x in table[0, :whole]] + pool[int(head):].tolist()
    assert sorted(rest) == list(range(P))


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_serving_within_a_budget(na, dtype):
    _serve(na, dtype, [(20, 30, 1), (1, 1, 50), (1, 1, 1), (1, 0, 1), (1, 20, 1), (9, 1, 1),
                       (1, 1, 1), (1, 1, 1), (1, 1, 1)], 60, 8)


def test_serving_within_a_budget_on_another_stream(na):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _serve(na, "bf16", [(20, 30), (1, 1), (40, 1), (1, 1), (1, 1), (5, 5)], 50, 4, prompt=32)
    s.synchronize()


def test_captured_steps_replay_with_new_lengths(na):
    """Attention, weights and eviction from two graphs: lengths and tokens change in place."""
    R, H, Hkv, D, page, most = 3, 4, 2, 64, 16, 20
    P = R * most
    table = torch.arange(P, dtype=torch.int32).reshape(R, most).cuda()
    table[1, :5] = table[0, :5]
    kp, vp = (_randn((P, Hkv, page, D), "bf16", i) for i in range(2))
    q = _randn((R, H, D), "bf16", 7)
    ctx, cu = _int([200, 180, 60]), _int([0, 1, 2, 3])
    groups, shared, first = _int([0, 2]), _int([80]), _int([80, 80, 0])
    weights = torch.rand(R, Hkv, most * page, device="cuda")
    free, head = torch.full((P,), -1, dtype=torch.int32, device="cuda"), _int([P])

    def step():
        w = weights.clone()
        out, lse = na.cache_shared_attention(q, kp, vp, table, ctx, cu, groups, shared, max_new=1,
                                             max_shared=100, max_own=200)
        na.cache_weights(q, lse, kp, table, ctx, cu, w, first=first, max_new=1, max_context=300)
        # (of copies, so that a replay finds the cache as it was)
        return (out, lse, w) + na.cache_evict(w, kp.clone(), vp.clone(), table, ctx, free, head,
                                              100, 9, first)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(step())
    for turn in range(6):
        ctx.copy_(torch.tensor([200 + 3 * turn, 90 + turn, 60 + 20 * turn]).int())
        shared.fill_(80 - turn)
        q.copy_(_randn(q.shape, "bf16", 100 + turn))
        weights.copy_(_weights(R, Hkv, most * page, turn))
        graphs[turn % 2].replay()
        got = [t.clone() for t in outs[turn % 2]]
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)
        want = ref.shared(q, kp, vp, table.tolist(), ctx.tolist(), [1] * R, [0, 2], [80 - turn],
                          WHOLE, 0, 0.125)
        plain.close(got[0], want[0], want[2], "out")


def test_two_calls_at_once_on_two_streams(na):
    streams = [torch.cuda.Stream() for _ in range(2)]
    own, new = [100, 400, 3], [1, 40, 2]
    want = _shared_check(na, own, new, [0, 3], [700], 4, 2, 64, 16, "bf16")
    for _ in range(3):
        got = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(_shared_check(na, own, new, [0, 3], [700], 4, 2, 64, 16, "bf16"))
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_calls_through_ctypes_agree(na, monkeypatch):
    import sys

    from paper_2403_04690_amd import sequence

    def run():
        w = _weights(2, 2, 300)
        return (_shared_check(na, [30, 5], [1, 2], [0, 2], [50], 4, 2, 64, 16, "fp16"),
                (_weights_check(na, [30, 50], [1, 2], 4, 2, 64, 16, "fp16"),),
                _evict_check(na, w, [300, 200], 64, 16, "bf16", 100, 10))

    fast = run()
    with monkeypatch.context() as m:
        m.setitem(sys.modules, "paper_2403_04690_amd._na_fast", None)
        m.setattr(sequence, "_bound", None)
        m.setattr(sequence, "_entry", {})
        slow = run()
        assert not any(isinstance(f, functools.partial) for f in sequence._entry.values())
    assert all(torch.equal(a, b) for x, y in zip(fast, slow) for a, b in zip(x, y))
