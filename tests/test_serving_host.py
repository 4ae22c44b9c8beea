"""Host-side checks of the cache operators for long contexts (no GPU needed, no kernel launched):
statuses of the C ABI, refusals of the binding, and the plain forms that the GPU tests compare
with."""
import ctypes
import math
import random

import pytest
import torch

import paper_2403_04690_amd as na
from paper_2403_04690_amd import sequence, serving
from tests import sequence_plain as plain
from tests import serving_plain as ref
from tests.test_sequence_host import (ALIGN, BAD_CACHE, DTYPE, FAKE, HEAD_DIM, NULL, OK, SHAPE,
                                      WORKSPACE, _cache)

BIG = 2 ** 63 - 1


@pytest.fixture(scope="module")
def lib():
    x = na.load_library()
    if not hasattr(x, "na_cache_evict"):
        pytest.skip("a library without the cache operators for long contexts")
    return sequence._library()


# ---------------------------------------------------------------- C ABI

def _shared(groups=2, max_shared=0, max_own=0, **cache):
    return sequence._SharedProblem(_cache(**cache), groups, max_shared, max_own)


def _attend(lib, p, work=FAKE, size=1 << 50, **ptr):
    names = ("q", "kp", "vp", "table", "ctx", "cu", "groups", "shared", "out", "lse")
    return lib.na_cache_shared_attention(p, *[ptr.get(n, FAKE) for n in names], work, size, None)


@pytest.mark.parametrize("change,status", BAD_CACHE + [
    ({"groups": -1}, SHAPE), ({"groups": 2 ** 24}, SHAPE), ({"groups": BIG}, SHAPE),
    ({"max_shared": -1}, SHAPE), ({"max_own": -1}, SHAPE),
    # row tiles of the join
    ({"requests": 2 ** 22, "kv_heads": 1}, SHAPE), ({"groups": 2 ** 23}, SHAPE)])
def test_shared_attention_rejects_before_launch(lib, change, status):
    assert _attend(lib, _shared(**change)) == status
    assert lib.na_cache_shared_attention_workspace(_shared(**change)) == 0


def test_shared_attention_pointers_and_workspace(lib):
    assert lib.na_cache_shared_attention(None, *[FAKE] * 11, 0, None) == NULL
    for name in ("q", "kp", "vp", "table", "ctx", "cu", "groups", "shared", "out", "lse"):
        assert _attend(lib, _shared(), **{name: None}) == NULL
        assert _attend(lib, _shared(), **{name: FAKE + 2}) == ALIGN
    need = lib.na_cache_shared_attention_workspace(_shared())
    assert need >= 2 * 5 * 4 * 65 * 4  # a part of the shared keys and one of the own, at least
    assert _attend(lib, _shared(), size=need - 1) == WORKSPACE
    assert _attend(lib, _shared(), work=None) == NULL
    assert _attend(lib, _shared(), work=FAKE + 8) == ALIGN
    for change in ({"requests": 0}, {"tokens": 0}, {"heads": 0, "kv_heads": 0}):
        assert _attend(lib, _shared(**change), q=None, work=None, size=0) == OK
    # no groups: their arrays are not looked at
    assert _attend(lib, _shared(groups=0), groups=None, shared=None, q=None) == NULL
    assert _attend(lib, _shared(max_shared=BIG, max_own=BIG, max_new=BIG), q=None) == NULL


def _weights(capacity=100, **cache):
    return sequence._WeightsProblem(_cache(**cache), capacity)


def _gather(lib, p, work=FAKE, size=1 << 50, **ptr):
    names = ("q", "lse", "kp", "table", "ctx", "cu", "first", "weights")
    return lib.na_cache_weights(p, *[ptr.get(n, FAKE) for n in names], work, size, None)


@pytest.mark.parametrize("change,status", [c for c in BAD_CACHE if "out" not in c[0]] + [
    ({"capacity": -1}, SHAPE), ({"capacity": BIG}, SHAPE), ({"capacity": 2 ** 38}, SHAPE),
    ({"requests": 2 ** 20, "max_pages": 1, "kv_heads": 1}, SHAPE)])
def test_weights_reject_before_launch(lib, change, status):
    assert _gather(lib, _weights(**change)) == status
    assert lib.na_cache_weights_workspace(_weights(**change)) == 0


def test_weights_pointers_and_workspace(lib):
    assert lib.na_cache_weights(None, *[FAKE] * 9, 0, None) == NULL
    for name in ("q", "lse", "kp", "table", "ctx", "cu", "weights"):
        assert _gather(lib, _weights(), **{name: None}) == NULL
        assert _gather(lib, _weights(), **{name: FAKE + 2}) == ALIGN
    assert _gather(lib, _weights(), first=FAKE + 2) == ALIGN
    # (the logsumexp and the weights by their element)
    assert _gather(lib, _weights(), lse=FAKE + 4, weights=FAKE + 4, q=None) == NULL
    # many rows over few keys are shared
    p = _weights(requests=1, tokens=4000, max_pages=8)
    need = lib.na_cache_weights_workspace(p)
    assert need > 0 and _gather(lib, p, size=need - 1) == WORKSPACE
    assert _gather(lib, p, work=None) == NULL and _gather(lib, p, work=FAKE + 2) == ALIGN
    # never more than 256 MiB
    for pages in (8, 2 ** 10, 2 ** 20, 2 ** 26):
        for requests in (1, 7, 60):
            if requests * pages < 2 ** 31:
                p = _weights(requests=requests, tokens=40000, max_pages=pages)
                assert lib.na_cache_weights_workspace(p) <= 2 ** 28
    for change in ({"requests": 0}, {"tokens": 0}, {"heads": 0, "kv_heads": 0}, {"capacity": 0}):
        assert _gather(lib, _weights(**change), q=None, work=None, size=0) == OK


def _evict(**change):
    f = dict(requests=3, kv_heads=2, head_dim=64, pages=8, page_size=16, max_pages=4, num_free=5,
             capacity=64, budget=20, recent=3, dtype=1)
    f.update(change)
    return sequence._EvictProblem(**f)


EVICT = ("weights", "ctx", "first", "table", "head", "free", "kp", "vp", "new_ctx", "new_weights",
         "kept", "new_head")


def _cut(lib, p, work=FAKE, size=1 << 50, **ptr):
    other = ("new_head", "new_ctx", "new_weights", "vp")
    ps = [ptr.get(n, FAKE + (64 if n in other else 0)) for n in EVICT]
    return lib.na_cache_evict(p, *ps, work, size, None)


@pytest.mark.parametrize("change,status", [
    ({"requests": -1}, SHAPE), ({"requests": BIG}, SHAPE), ({"kv_heads": 0}, SHAPE),
    ({"kv_heads": -2}, SHAPE), ({"kv_heads": BIG}, SHAPE), ({"head_dim": 48}, HEAD_DIM),
    ({"dtype": 3}, DTYPE), ({"pages": -1}, SHAPE), ({"page_size": 8}, SHAPE),
    ({"page_size": 48}, SHAPE), ({"max_pages": -1}, SHAPE), ({"max_pages": 2 ** 27}, SHAPE),
    ({"num_free": -1}, SHAPE), ({"num_free": 2 ** 30}, SHAPE), ({"capacity": -1}, SHAPE),
    ({"capacity": 2 ** 39}, SHAPE), ({"budget": 0}, SHAPE), ({"budget": 2 ** 30}, SHAPE),
    ({"recent": -1}, SHAPE), ({"requests": 2 ** 19, "max_pages": 1}, SHAPE),
    ({"page_size": 2 ** 20, "max_pages": 1, "kv_heads": 64}, SHAPE)])
def test_evict_rejects_before_launch(lib, change, status):
    assert _cut(lib, _evict(**change)) == status
    assert lib.na_cache_evict_workspace(_evict(**change)) == 0


def test_evict_pointers_and_workspace(lib):
    assert lib.na_cache_evict(None, *[FAKE] * 13, 0, None) == NULL
    for name in EVICT:
        if name != "first":
            assert _cut(lib, _evict(), **{name: None}) == NULL
        assert _cut(lib, _evict(), **{name: FAKE + 2}) == ALIGN
    for name in ("kp", "vp"):
        assert _cut(lib, _evict(), **{name: FAKE + 8}) == ALIGN
    assert _cut(lib, _evict(), new_head=FAKE) == SHAPE
    assert _cut(lib, _evict(), new_ctx=FAKE) == SHAPE
    assert _cut(lib, _evict(), new_weights=FAKE) == SHAPE
    assert _cut(lib, _evict(), vp=FAKE) == SHAPE
    need = lib.na_cache_evict_workspace(_evict())
    assert need == 3 * 2 * (2 * 20 + 2) * 4
    assert _cut(lib, _evict(), size=need - 1) == WORKSPACE
    assert _cut(lib, _evict(), work=None) == NULL and _cut(lib, _evict(), work=FAKE + 2) == ALIGN
    assert _cut(lib, _evict(recent=BIG), work=None) == NULL  # (valid: the pointer is refused)


def test_problems_are_laid_out_as_in_c(lib):
    assert ctypes.sizeof(sequence._SharedProblem) == ctypes.sizeof(sequence._CacheProblem) + 24
    assert ctypes.sizeof(sequence._WeightsProblem) == ctypes.sizeof(sequence._CacheProblem) + 8
    assert ctypes.sizeof(sequence._EvictProblem) == 88


# ---------------------------------------------------------------- binding

def _ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def test_binding_refuses_before_launch(lib):
    q, kp = torch.zeros(3, 4, 32), torch.zeros(5, 2, 16, 32)
    table, ctx, cu = torch.zeros(2, 4, dtype=torch.int32), _ints(3, 4), _ints(0, 1, 3)
    lse, w = torch.zeros(3, 4), torch.zeros(2, 2, 64)
    args = (q, kp, kp, table, ctx, cu)
    with pytest.raises(ValueError, match="GPU"):
        na.cache_shared_attention(*args, _ints(0, 2), _ints(5))
    with pytest.raises(ValueError, match="GPU"):
        na.cache_weights(q, lse, kp, table, ctx, cu, w)
    with pytest.raises(ValueError, match="GPU"):
        na.cache_evict(w, kp, kp, table, ctx, _ints(0), _ints(0), 10)
    for bad, match in (((q[0],) + args[1:], "tokens, heads"), ((q[:, :3],) + args[1:], "multiple"),
                       ((q, kp, kp[:, :1], table, ctx, cu), "alike"),
                       (args[:5] + (cu[:2],), "cu_new"), (args[:3] + (table[:1], ctx, cu), "page_table")):
        with pytest.raises(ValueError, match=match):
            na.cache_shared_attention(*bad, _ints(0, 2), _ints(5))
    with pytest.raises(ValueError, match="lse"):
        na.cache_weights(q, None, kp, table, ctx, cu, w)


def _meta(t, device):
    return t.shape, t.stride(), t.dtype, torch.device(device)


def test_plans_check_what_belongs_together(lib):
    """The checks behind the device's, with the metas of tensors that would be on a GPU."""
    gpu = "cuda:0"
    q, kp = _meta(torch.zeros(3, 4, 32), gpu), _meta(torch.zeros(5, 2, 16, 32), gpu)
    table, ctx = _meta(torch.zeros(2, 4, dtype=torch.int32), gpu), _meta(_ints(3, 4), gpu)
    cu, groups, shared = (_meta(_ints(*x), gpu) for x in ((0, 1, 3), (0, 2), (5,)))
    lse, w = _meta(torch.zeros(3, 4), gpu), _meta(torch.zeros(2, 2, 64), gpu)
    cache = (q, kp, kp, table, ctx, cu, None, None)

    def plan(groups=groups, shared=shared, **kw):
        a = {"max_new": None, "max_shared": None, "max_own": None, **kw}
        return serving._shared_plan.__wrapped__(None, 0, None, a["max_new"], a["max_shared"],
                                                a["max_own"], cache + (groups, shared))

    assert plan()[2] > 0
    for bad, error in (
            ({"groups": _meta(_ints(0, 1, 2), gpu)}, ValueError),
            ({"shared": _meta(torch.zeros(1, dtype=torch.int64), gpu)}, TypeError),
            ({"shared": _meta(_ints(5), "cuda:1")}, ValueError),
            ({"groups": _meta(_ints(0, 0, 0, 0)[::2], gpu)}, ValueError),
            ({"max_own": -1}, ValueError), ({"max_shared": -1}, ValueError)):
        with pytest.raises(error):
            plan(**bad)

    def gather(lse=lse, w=w, first=None):
        return serving._weights_plan.__wrapped__(None, 0, None, None, None,
                                                 (q, lse, kp, table, ctx, cu, w, first))

    assert gather()[2] == 0
    assert gather(first=ctx)[0].capacity == 64
    for bad, error in (({"w": _meta(torch.zeros(2, 2, 64).half(), gpu)}, TypeError),
                       ({"w": _meta(torch.zeros(2, 4, 64), gpu)}, ValueError),
                       ({"w": _meta(torch.zeros(2, 2, 128)[:, :, ::2], gpu)}, ValueError),
                       ({"w": _meta(torch.zeros(2, 2, 64), "cpu")}, ValueError),
                       ({"lse": _meta(torch.zeros(3, 3), gpu)}, ValueError),
                       ({"first": _meta(_ints(1), gpu)}, ValueError),
                       ({"first": _meta(torch.zeros(2), gpu)}, TypeError)):
        with pytest.raises(error):
            gather(**bad)

    free, head = _meta(_ints(1, 2, 3), gpu), _meta(_ints(0), gpu)

    def cut(budget=10, recent=0, w=w, kp=kp, free=free, head=head, first=None):
        return serving._evict_plan.__wrapped__(budget, recent,
                                               (w, kp, kp, table, ctx, free, head, first))

    assert cut()[2] == 2 * 2 * 22 * 4
    for bad, error in (({"budget": 0}, ValueError), ({"recent": -1}, ValueError),
                       ({"w": _meta(torch.zeros(2, 1, 64), gpu)}, ValueError),
                       ({"kp": _meta(torch.zeros(5, 2, 16, 64)[..., ::2], gpu)}, ValueError),
                       ({"kp": _meta(torch.zeros(5, 2, 16, 32).double(), gpu)}, TypeError),
                       ({"free": _meta(torch.zeros(2, 2, dtype=torch.int32), gpu)}, ValueError),
                       ({"head": _meta(_ints(1, 2), gpu)}, ValueError),
                       ({"first": _meta(_ints(1, 2), "cuda:1")}, ValueError)):
        with pytest.raises(error):
            cut(**bad)


def test_evict_plans_refuse_what_the_library_refuses(lib):
    """Before the call allocates outputs of such sizes."""
    gpu = "cuda:0"
    kp, w = _meta(torch.zeros(5, 2, 16, 32), gpu), _meta(torch.zeros(2, 2, 64), gpu)
    table, ctx = _meta(torch.zeros(2, 4, dtype=torch.int32), gpu), _meta(_ints(3, 4), gpu)
    free, head = _meta(_ints(1, 2, 3), gpu), _meta(_ints(0), gpu)

    def cut(budget, kp=kp, w=w):
        return serving._evict_plan.__wrapped__(budget, 0, (w, kp, kp, table, ctx, free, head, None))

    assert cut(2 ** 30 - 1)[0].budget == 2 ** 30 - 1
    odd = torch.Size((5, 2, 24, 32)), (2 * 24 * 32, 24 * 32, 32, 1), torch.float32, kp[3]
    for bad, status in (({"budget": 2 ** 30}, SHAPE), ({"budget": 2 ** 40}, SHAPE),
                        ({"budget": 9, "kp": odd}, SHAPE),
                        ({"budget": 9, "kp": _meta(torch.zeros(5, 2, 16, 48), gpu)}, HEAD_DIM)):
        with pytest.raises(na.NAError) as e:
            cut(**bad)
        assert e.value.status == status


# ---------------------------------------------------------------- the plain forms

def test_plain_shared_is_plain_attention_where_nothing_is_shared():
    gen = torch.Generator().manual_seed(0)
    kp, vp = (torch.randn((6, 2, 16, 8), generator=gen) for _ in range(2))
    q = torch.randn((4, 4, 8), generator=gen)
    table, context, new = [[3, 1, -1], [0, 5, 2]], [10, 33], [1, 3]
    a = plain.cache(q, kp, vp, table, context, new, 9, 2, 0.3)
    b = ref.shared(q, kp, vp, table, context, new, [0], [], 9, 2, 0.3)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # and where the shared tokens are the request's own
    c = ref.shared(q, kp, vp, table, context, new, [0, 1, 2], [20, 20], 9, 2, 0.3)
    assert torch.equal(a[0], c[0])


def test_plain_weights_are_the_sums_of_a_softmax():
    gen = torch.Generator().manual_seed(1)
    kp = torch.randn((4, 1, 16, 8), generator=gen)
    q = torch.randn((3, 2, 8), generator=gen)
    lse = ref.shared(q, kp, kp, [[2, 0]], [20], [3], [0], [], 2 ** 31, 0, 0.3)[1]
    w, _ = ref.weights(q, lse, kp, [[2, 0]], [20], [3], torch.zeros(1, 1, 30), 2 ** 31, 0, 0.3)
    assert abs(float(w.sum()) - 6) < 1e-6 and float(w[0, 0, 23:].abs().max()) == 0


def test_plain_eviction_keeps_what_it_should():
    rng = random.Random(0)
    for _ in range(50):
        n, budget = rng.randint(1, 60), rng.randint(1, 40)
        recent, first = rng.randint(0, 45), rng.randint(0, 45)
        w = torch.tensor([rng.choice((0.0, 1.0, rng.random())) for _ in range(60)]).reshape(1, 1, 60)
        kp = torch.arange(4 * 16, dtype=torch.float32).reshape(4, 1, 16, 1).repeat(1, 1, 1, 2)
        after, new_w, kept, head, free, nk, nv = ref.evict(w, kp, kp, [[0, 1, 2, 3]], [n], [-1] * 4, 4,
                                                           budget, recent, [first])
        m = min(n, budget)
        ids = kept[0, 0, :m].tolist()
        assert after == [m] and len(set(ids)) == m and kept[0, 0, m:].eq(-1).all()
        assert nk.reshape(64, 2)[:m, 0].tolist() == [float(i) for i in ids]
        assert torch.equal(new_w[0, 0, :m], w[0, 0, ids]) and new_w[0, 0, m:].eq(0).all()
        if n > budget:
            f = min(first, budget)
            last = min(recent, budget - f)
            assert ids[:f] == list(range(f)) and ids[m - last:] == list(range(n - last, n))
            gone = sorted(set(range(n)) - set(ids))
            stay = sorted(set(ids) - set(range(f)) - set(range(n - last, n)))
            if gone and stay:
                # no token that went comes before one that stayed
                assert max((float(w[0, 0, i]), -i) for i in gone) < min(
                    (float(w[0, 0, i]), -i) for i in stay)
            assert head == 4 - (-(-n // 16) - -(-budget // 16))
            assert free[head:] == list(range(-(-budget // 16), -(-n // 16)))
        else:
            assert ids == list(range(n)) and head == 4 and math.isclose(float(nk.sum()), float(kp.sum()))
