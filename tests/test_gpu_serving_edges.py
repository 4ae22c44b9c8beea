"""The cache operators for long contexts at the edges of their inputs: values that are not finite,
positions that are far apart."""
import math

import pytest
import torch

from tests import sequence_plain as plain
from tests import serving_plain as ref
from tests.test_gpu_serving import (WHOLE, _int, _offsets, _randn, _tables,  # noqa: F401
                                    na)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- values that are not finite

class _Served:
    """Requests 0 and 1 share 100 tokens, request 2 is in no group; every request lists the shared
    pages, so that cache_attention reads the same keys."""

    def __init__(self, na, dtype, D, new, own=(40, 470, 20), H=4, Hkv=2, page=16, scale=None):
        self.na, self.scale, self.new = na, scale, new
        self.context = [own[0] + 100, own[1] + 100, own[2]]
        table, P, _ = _tables(self.context, new, page, [0, 2], [96])
        self.table = table
        self.kp, self.vp = (_randn((P, Hkv, page, D), dtype, 1 + i) for i in range(2))
        # (the page in which the shared tokens end is request 0's and, copied, request 1's)
        for t in (self.kp, self.vp):
            t[table[1][6], :, :4] = t[table[0][6], :, :4]
        self.q = _randn((sum(new), H, D), dtype, 3)
        self.page, self.G = page, H // Hkv

    def put(self, pages, r, j, head, value):
        """The row of position j of request r; shared ones of both that have them."""
        for x in ((0, 1) if r < 2 and j < 100 else (r,)):
            pages[self.table[x][j // self.page], head, j % self.page] = value

    def shared(self, **hints):
        return self.na.cache_shared_attention(
            self.q, self.kp, self.vp, torch.tensor(self.table).int().cuda(), _int(self.context),
            _offsets(self.new), _int([0, 2]), _int([100]), None, 0, self.scale, **hints)

    def attend(self):
        return self.na.cache_attention(
            self.q, self.kp, self.vp, torch.tensor(self.table).int().cuda(), _int(self.context),
            _offsets(self.new), None, 0, self.scale)[0]


FORMS = [([1, 1, 1], {"max_new": 1, "max_shared": 100, "max_own": 500}), ([40, 3, 2], {}),
         ([1, 1, 1], {"max_new": 1, "max_shared": 1, "max_own": 1}),
         ([90, 130, 1], {"max_new": 130, "max_shared": 100, "max_own": 1})]


@pytest.mark.parametrize("dtype,D", [("fp32", 32), ("fp16", 64), ("bf16", 128), ("fp32", 128)])
@pytest.mark.parametrize("new,hints", FORMS)
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("request_,j", [(0, 33), (0, 120), (1, 400), (1, 98), (2, 7)])
def test_a_key_that_is_not_finite_shows_in_the_rows_that_see_it(na, dtype, D, new, hints, value,
                                                               request_, j):
    x = _Served(na, dtype, D, new)
    out, lse = x.shared(**hints)
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all())
    x.put(x.kp, request_, j, 1, value)  # (of head 1: heads 2 and 3 of the queries)
    bad, bad_lse = x.shared(**hints)
    hit = torch.zeros(sum(new), 4, dtype=torch.bool)
    at = [sum(new[:r]) for r in range(4)]
    for r in ((0, 1) if request_ < 2 and j < 100 else (request_,)):
        hit[at[r]:at[r + 1], 2:] = True
    hit = hit.cuda()
    assert not bool(bad.isfinite()[hit].any()) and not bool(bad_lse.isfinite()[hit].any())
    assert torch.equal(bad[~hit], out[~hit]) and torch.equal(bad_lse[~hit], lse[~hit])
    assert torch.equal(x.attend().isfinite(), bad.isfinite())


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("new,hints", FORMS)
def test_every_form_shows_keys_queries_and_values_that_are_not_finite(na, dtype, D, new, hints):
    x = _Served(na, dtype, D, new)
    want, want_lse = x.shared(**hints)
    keys, values, query = x.kp.clone(), x.vp.clone(), x.q.clone()
    for j in (33, 120):
        x.put(x.kp, 0, j, 0, math.nan)
        out, lse = x.shared(**hints)
        assert not bool(out[0, :2].isfinite().any()) and not bool(lse[0, :2].isfinite().any())
        assert torch.equal(out[0, 2:], want[0, 2:]) and torch.equal(lse[0, 2:], want_lse[0, 2:])
        x.kp.copy_(keys)
        x.put(x.vp, 0, j, 0, math.inf)
        out, lse = x.shared(**hints)
        assert not bool(out[0, :2].isfinite().any()) and torch.equal(lse, want_lse)
        assert torch.equal(out[0, 2:], want[0, 2:])
        x.vp.copy_(values)
    x.q[0, 0, 3] = math.nan
    out, lse = x.shared(**hints)
    assert not bool(out[0, 0].isfinite().any()) and not bool(lse[0, 0].isfinite())
    out[0, 0], lse[0, 0] = want[0, 0], want_lse[0, 0]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    x.q.copy_(query)
    out, lse = x.shared(**hints)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype,D", [("fp32", 32), ("fp16", 64), ("bf16", 128)])
@pytest.mark.parametrize("new,hints", FORMS)
def test_a_query_that_is_not_finite_shows_in_its_row(na, dtype, D, new, hints):
    x = _Served(na, dtype, D, new)
    out, lse = x.shared(**hints)
    hit = torch.zeros(sum(new), 4, dtype=torch.bool, device="cuda")
    for t, h, value in ((0, 1, math.nan), (sum(new) - 1, 3, math.inf), (new[0], 2, math.nan)):
        x.q[t, h, 5:7] = value
        hit[t, h] = True
    x.q[sum(new) - 1, 3, 6] = -math.inf
    bad, bad_lse = x.shared(**hints)
    nan = torch.zeros_like(hit)
    nan[0, 1] = nan[new[0], 2] = True
    assert not bool(bad.isfinite()[nan].any()) and not bool(bad_lse.isfinite()[nan].any())
    # (infinite scores of both signs are among the keys of the third one)
    assert not bool(bad.isfinite()[hit].any()) and not bool(bad_lse.isfinite()[hit].any())
    assert torch.equal(bad[~hit], out[~hit]) and torch.equal(bad_lse[~hit], lse[~hit])


@pytest.mark.parametrize("new,hints", FORMS)
def test_scores_that_overflow_show(na, new, hints):
    """Finite queries and keys whose products are beyond fp32."""
    for j in (33, 120):
        x = _Served(na, "bf16", 64, new)
        x.put(x.kp, 0, j, 0, 1e30)
        x.q[0, 0] = 1e30
        out, lse = x.shared(**hints)
        assert not bool(out[0, 0].isfinite().any()) and not bool(lse[0, 0].isfinite())
        assert not bool(x.attend()[0, 0].isfinite().any())


@pytest.mark.parametrize("dtype,D", [("fp32", 64), ("fp16", 128), ("bf16", 32)])
@pytest.mark.parametrize("new,hints", FORMS)
@pytest.mark.parametrize("scale", [None, 400.0])
def test_values_that_are_not_finite_show_where_cache_attention_has_them(na, dtype, D, new, hints, scale):
    """In their column, with a weight that vanishes against the other keys' too."""
    x = _Served(na, dtype, D, new, scale=scale)
    out, lse = x.shared(**hints)
    places = [(0, 33, 5, math.nan), (1, 400, 9, math.nan), (2, 7, 3, math.nan), (0, 120, 1, math.nan)]
    for r, j, d, value in places:
        for y in ((0, 1) if r < 2 and j < 100 else (r,)):
            x.vp[x.table[y][j // 16], 1, j % 16, d] = value
    bad, bad_lse = x.shared(**hints)
    assert torch.equal(bad_lse, lse)
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    at = [sum(new[:r]) for r in range(4)]
    for r, j, d, _ in places:
        for y in ((0, 1) if r < 2 and j < 100 else (r,)):
            hit[at[y]:at[y + 1], 2:, d] = True
    assert not bool(bad.isfinite()[hit].any()) and torch.equal(bad[~hit], out[~hit])
    assert torch.equal(x.attend().isfinite(), bad.isfinite())


# ---------------------------------------------------------------- positions far apart

@pytest.mark.parametrize("dtype,D", [("fp32", 32), ("bf16", 128)])
@pytest.mark.parametrize("new,hints", [([1, 1, 2], {"max_new": 2}), ([60, 3, 80], {})])
@pytest.mark.parametrize("W", [None, 2 ** 31 - 1, 2 ** 31 - 129, 2 ** 30, 4000, 130])
def test_rows_of_a_group_that_stand_far_apart(na, dtype, D, new, hints, W):
    """A row before most of the keys that its group shares, beside rows behind all of them: its
    distances from those keys, less the widest window, are beyond 32 bits."""
    context, shared, page = [0, 5000, 300], 4900, 64
    most = [max(c + n, shared) for c, n in zip(context, new)]
    made, P, _ = _tables(most, [0, 0, 0], page, [0, 3], [shared])
    kp, vp = (_randn((P, 2, page, D), dtype, 1 + i) for i in range(2))
    q = _randn((sum(new), 4, D), dtype, 3)
    w = WHOLE if W is None else W
    want = ref.shared(q, kp, vp, made, context, new, [0, 3], [shared], w, 3, D ** -0.5)
    out, lse = na.cache_shared_attention(
        q, kp, vp, torch.tensor(made).int().cuda(), _int(context), _offsets(new), _int([0, 3]),
        _int([shared]), W, 3, **hints)
    plain.close(out, want[0], want[2], "out")
    plain.close(lse, want[1], want[3], "lse")


# ---------------------------------------------------------------- memory that held something else

def _used_before(value, dtype):
    """What the allocator hands out next held this."""
    free = [torch.full((n,), value, dtype=dtype, device="cuda")
            for n in (2 ** 20, 2 ** 24) + (2 ** 14,) * 8 + (2 ** 17,) * 4]
    del free


@pytest.mark.parametrize("dtype,D", [("fp32", 64), ("bf16", 128)])
@pytest.mark.parametrize("new", [[1] * 40, [70, 3] + [1] * 38])
def test_results_do_not_depend_on_what_workspaces_held(na, dtype, D, new):
    """Requests with and without a group, many splits of their keys; other calls in between."""
    R, H, Hkv, page = 40, 8, 2, 64
    cu, shared = [0, 30, 36], [3000, 90]
    own = [(97 * r) % 600 for r in range(R)]
    of = ref.groups_of(R, cu, shared)
    context = [c + s for c, (_, s) in zip(own, of)]
    table, P, _ = _tables(context, new, page, cu, shared)
    kp, vp = (_randn((P, Hkv, page, D), dtype, 1 + i) for i in range(2))
    q = _randn((sum(new), H, D), dtype, 3)
    t, ctx, off = torch.tensor(table).int().cuda(), _int(context), _offsets(new)
    hints = {"max_new": max(new)}
    first = _int([s // 2 for _, s in of])
    # (eviction: of requests that share no pages)
    lens = [1 + (211 * r) % 1900 for r in range(R)]
    apart, P2, _ = _tables(lens, [0] * R, page, [0], [], seed=1)
    t2, pool = torch.tensor(apart).int().cuda(), _randn((P2, Hkv, page, D), dtype, 7)
    weights = torch.rand((R, Hkv, t2.shape[1] * page), device="cuda").mul(40).round()

    def run():
        out, lse = na.cache_shared_attention(q, kp, vp, t, ctx, off, _int(cu), _int(shared),
                                             max_shared=3000, max_own=700, **hints)
        w = torch.zeros(R, Hkv, t.shape[1] * page, device="cuda")
        na.cache_weights(q, lse, kp, t, ctx, off, w, first=first, max_context=3700, **hints)
        free, head = torch.full((P2,), -1, dtype=torch.int32, device="cuda"), _int([P2])
        k, v = pool.clone(), -pool
        cut = na.cache_evict(weights, k, v, t2, _int(lens), free, head, 500, 50, first // 4)
        return (out, lse, w, k, v, free) + cut

    want = run()
    for value, kind in ((math.nan, torch.float32), (-1, torch.int32), (2 ** 30, torch.int32),
                        (math.inf, torch.float32)):
        _used_before(value, kind)
        na.cache_shared_attention(-q, vp, kp, t, ctx, off, _int(cu), _int(shared))
        for a, b in zip(run(), want):
            assert torch.equal(a, b)
