"""Host-side checks of the sequence operators (no GPU needed, no kernel launched): the C ABI's
statuses and the binding's refusals come before any launch; the plain forms that the GPU tests
compare with are pinned here."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2403_04690_amd as na
from paper_2403_04690_amd import sequence
from tests import sequence_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, KERNEL, HEAD_DIM, DTYPE, ALIGN, SCALE, WORKSPACE = 0, 1, 3, 4, 7, 8, 9, 12, 15
FAKE = 0x10000  # aligned, never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    raw = na.load_library()
    if not hasattr(raw, "na_sink_forward"):
        pytest.skip("a library without the sequence operators")
    return sequence._library()


def test_library_exports_every_declared_symbol(lib):
    text = open(os.path.join(ROOT, "include", "na_seq.h")).read()
    names = set(re.findall(r"\b(na_[a-z_]+)\s*\(", re.sub(r"/\*.*?\*/", "", text, flags=re.S)))
    assert {"na_sink_forward", "na_sink_backward", "na_sink_backward_workspace", "na_cache_tables", "na_cache_write", "na_cache_attention",
            "na_cache_attention_workspace"} <= names
    for name in names:
        assert hasattr(lib, name), name


def test_workspace_status_has_a_text(lib):
    assert b"workspace" in lib.na_status_string(WORKSPACE)


# ---------------------------------------------------------------- C ABI

STRIDED = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")


def _sink(batch=2, heads=4, kv_heads=2, tokens=10, head_dim=64, kernel_size=3, sinks=1, dtype=1,
          scale=0.125, **strides):
    p = sequence._SinkProblem(batch, heads, kv_heads, tokens, head_dim, kernel_size, sinks)
    for name in STRIDED:
        h = kv_heads if name in ("k", "v", "dk", "dv") else heads
        s = strides.get(name, (h * tokens * head_dim, tokens * head_dim, head_dim))
        setattr(p, name, sequence._Strides(*s))
    p.dtype, p.scale = dtype, scale
    return p


def _forward(lib, p, q=FAKE, k=FAKE, v=FAKE, lengths=None, out=FAKE, lse=FAKE):
    return lib.na_sink_forward(p, q, k, v, lengths, out, lse, None)


BAD_SINK = [
    ({"batch": -1}, SHAPE), ({"heads": -4}, SHAPE), ({"tokens": -1}, SHAPE),
    ({"kv_heads": 3}, SHAPE), ({"kv_heads": 0}, SHAPE), ({"sinks": -1}, SHAPE),
    ({"kernel_size": 0}, KERNEL), ({"kernel_size": -2 ** 62}, KERNEL),
    ({"head_dim": 80}, HEAD_DIM), ({"dtype": 3}, DTYPE), ({"dtype": -1}, DTYPE),
    ({"scale": math.inf}, SCALE), ({"scale": math.nan}, SCALE),
    ({"tokens": 2 ** 30}, SHAPE), ({"tokens": 2 ** 62}, SHAPE), ({"batch": 2 ** 62}, SHAPE),
    ({"heads": 2 ** 40, "kv_heads": 1}, SHAPE), ({"batch": 2 ** 24}, SHAPE),
    ({"tokens": 2 ** 29, "heads": 4, "kv_heads": 1}, SHAPE),
    # a token stride that is no multiple of 16 bytes; one that is negative; one too large
    ({"q": (2560, 640, 60)}, SHAPE), ({"k": (1280, 640, -64)}, SHAPE),
    ({"v": (1280, 640, 2 ** 26)}, SHAPE), ({"v": (2 ** 62, 640, 64)}, SHAPE),
    ({"q": (2559, 640, 64)}, SHAPE),
]


@pytest.mark.parametrize("change,status", BAD_SINK)
def test_sink_forward_rejects_before_launch(lib, change, status):
    assert _forward(lib, _sink(**change)) == status


@pytest.mark.parametrize("out", [(0, 640, 64), (2560, 0, 64), (2560, 640, 0), (2560, 640, 32),
                                 (640, 640, 64), (2552, 640, 64)])
def test_outputs_must_not_overlap_themselves(lib, out):
    assert _forward(lib, _sink(out=out)) == SHAPE


def test_sink_forward_pointers(lib):
    assert lib.na_sink_forward(None, FAKE, FAKE, FAKE, None, FAKE, FAKE, None) == NULL
    for name in ("q", "k", "v", "out", "lse"):
        assert _forward(lib, _sink(), **{name: None}) == NULL
        assert _forward(lib, _sink(), **{name: FAKE + 8}) == ALIGN
    assert _forward(lib, _sink(), lengths=FAKE + 2) == ALIGN
    # nothing to do: pointers are not looked at
    for change in ({"batch": 0}, {"tokens": 0}, {"heads": 0, "kv_heads": 0}):
        assert _forward(lib, _sink(**change), q=None, out=FAKE + 2) == OK


def _backward(lib, p, work=FAKE, size=1 << 40, lengths=None, **ptr):
    names = ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv")
    ps = [ptr.get(n, FAKE) for n in names]
    return lib.na_sink_backward(p, *ps[:3], lengths, *ps[3:], work, size, None)


@pytest.mark.parametrize("change,status", BAD_SINK + [
    ({"dout": (2560, 640, 60)}, SHAPE), ({"dq": (2560, 640, 0)}, SHAPE),
    ({"dk": (0, 640, 64)}, SHAPE), ({"dv": (1280, 640, 32)}, SHAPE)])
def test_sink_backward_rejects_before_launch(lib, change, status):
    assert _backward(lib, _sink(**change)) == status
    assert lib.na_sink_backward_workspace(_sink(**change)) == 0


def test_sink_backward_pointers_and_workspace(lib):
    assert lib.na_sink_backward(None, *[FAKE] * 11, 0, None) == NULL
    for name in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"):
        assert _backward(lib, _sink(), **{name: None}) == NULL
        assert _backward(lib, _sink(), **{name: FAKE + 4}) == ALIGN
    assert _backward(lib, _sink(), lengths=FAKE + 2) == ALIGN
    need = lib.na_sink_backward_workspace(_sink())
    assert need >= 2 * 2 * 4 * 10 * 4  # two fp32 a row at least
    assert _backward(lib, _sink(), size=need - 1) == WORKSPACE
    assert _backward(lib, _sink(), work=None) == NULL
    assert _backward(lib, _sink(), work=FAKE + 8) == ALIGN
    for change in ({"batch": 0}, {"tokens": 0}, {"heads": 0, "kv_heads": 0}):
        assert _backward(lib, _sink(**change), q=None, work=None, size=0) == OK


def _cache(requests=3, tokens=5, heads=4, kv_heads=2, head_dim=64, pages=8, page_size=16,
           max_pages=4, kernel_size=100, sinks=0, max_new=0, max_context=0, dtype=1, scale=0.1,
           q=None, k=None, v=None, out=None):
    p = sequence._CacheProblem(requests, tokens, heads, kv_heads, head_dim, pages, page_size,
                               max_pages, kernel_size, sinks, max_new, max_context)
    for name, s, h in (("q", q, heads), ("k", k, kv_heads), ("v", v, kv_heads), ("out", out, heads)):
        setattr(p, name, sequence._Strides(*(s or (0, head_dim, h * head_dim))))
    p.dtype, p.scale = dtype, scale
    return p


def _attend(lib, p, q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, ctx=FAKE, cu=FAKE, out=FAKE, lse=FAKE,
            work=None, size=0):
    return lib.na_cache_attention(p, q, kp, vp, table, ctx, cu, out, lse, work, size, None)


BAD_CACHE = [
    ({"requests": -1}, SHAPE), ({"tokens": -1}, SHAPE), ({"pages": -1}, SHAPE),
    ({"page_size": 8}, SHAPE), ({"page_size": 24}, SHAPE), ({"page_size": 0}, SHAPE),
    ({"page_size": -16}, SHAPE), ({"page_size": 2 ** 21}, SHAPE), ({"max_pages": -1}, SHAPE),
    ({"max_pages": 2 ** 29}, SHAPE), ({"requests": 2 ** 23, "max_pages": 256}, SHAPE),
    ({"kv_heads": 3}, SHAPE), ({"head_dim": 96}, HEAD_DIM), ({"dtype": 7}, DTYPE),
    ({"scale": math.nan}, SCALE), ({"kernel_size": 0}, KERNEL), ({"sinks": -3}, SHAPE),
    ({"max_new": -1}, SHAPE), ({"max_context": -1}, SHAPE), ({"tokens": 2 ** 30}, SHAPE),
    ({"tokens": 2 ** 29}, SHAPE), ({"q": (0, 64, 250)}, SHAPE), ({"out": (0, 64, 64)}, SHAPE),
]


@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_cache_attention_rejects_before_launch(lib, change, status):
    assert _attend(lib, _cache(**change)) == status
    assert lib.na_cache_attention_workspace(_cache(**change)) == 0


def test_cache_attention_pointers_and_workspace(lib):
    assert lib.na_cache_attention(None, *[FAKE] * 9, 0, None) == NULL
    for name in ("q", "kp", "vp", "table", "ctx", "cu", "out", "lse"):
        assert _attend(lib, _cache(), **{name: None}) == NULL
        assert _attend(lib, _cache(), **{name: FAKE + 2}) == ALIGN
    # one request over a long context: its keys are split, which takes a workspace
    p = _cache(requests=1, tokens=1, max_pages=2 ** 12, kernel_size=2 ** 31 - 1)
    need = lib.na_cache_attention_workspace(p)
    assert need > 0
    assert _attend(lib, p, work=FAKE, size=need - 1) == WORKSPACE
    assert _attend(lib, p, work=None, size=need) == NULL
    assert _attend(lib, p, work=FAKE + 8, size=need) == ALIGN
    # a short window never is
    assert lib.na_cache_attention_workspace(_cache(requests=1, tokens=1, max_pages=2 ** 12)) == 0
    for change in ({"requests": 0}, {"tokens": 0}, {"heads": 0, "kv_heads": 0}):
        assert _attend(lib, _cache(**change), q=None) == OK


def test_extreme_counts_do_not_overflow(lib):
    big = 2 ** 63 - 1
    for p in (_cache(kernel_size=big), _cache(sinks=big, kernel_size=big),
              _cache(max_new=big, max_context=big)):
        assert _attend(lib, p, q=None) == NULL  # (valid: the pointer is what is refused)
    assert _forward(lib, _sink(kernel_size=big, sinks=big), q=None) == NULL
    assert _backward(lib, _sink(kernel_size=big, sinks=big), q=None) == NULL
    assert _backward(lib, _sink(sinks=big), q=None) == NULL
    for name in ("requests", "tokens", "heads", "kv_heads", "pages", "page_size", "max_pages"):
        assert _attend(lib, _cache(**{name: big})) == SHAPE
    for name in ("batch", "heads", "kv_heads", "tokens"):
        assert _forward(lib, _sink(**{name: big})) == SHAPE


def _write(lib, p, k=FAKE, v=FAKE, slots=FAKE, kp=FAKE, vp=FAKE):
    return lib.na_cache_write(p, k, v, slots, kp, vp, None)


@pytest.mark.parametrize("change,status", [
    ({"tokens": -1}, SHAPE), ({"kv_heads": -1}, SHAPE), ({"pages": -1}, SHAPE),
    ({"page_size": 40}, SHAPE), ({"head_dim": 8}, HEAD_DIM), ({"dtype": 9}, DTYPE),
    ({"k": (0, 60, 128)}, SHAPE), ({"v": (0, 64, -128)}, SHAPE),
    ({"tokens": 2 ** 29, "kv_heads": 2}, SHAPE), ({"tokens": 2 ** 63 - 1}, SHAPE),
])
def test_cache_write_rejects_before_launch(lib, change, status):
    assert _write(lib, _cache(**change)) == status


def test_cache_write_pointers(lib):
    assert lib.na_cache_write(None, *[FAKE] * 5, None) == NULL
    for name in ("k", "v", "slots", "kp", "vp"):
        assert _write(lib, _cache(), **{name: None}) == NULL
        assert _write(lib, _cache(), **{name: FAKE + 4}) == ALIGN
    assert _write(lib, _cache(tokens=0), k=None) == OK


def _tables(lib, requests=2, tokens=5, page_size=16, max_pages=4, num_free=3, **ptr):
    names = ("context", "new", "free", "head", "table", "cu", "slots", "positions", "new_head")
    ps = [ptr.get(n, FAKE + (64 if n == "new_head" else 0)) for n in names]
    return lib.na_cache_tables(requests, tokens, page_size, max_pages, num_free, *ps, None)


@pytest.mark.parametrize("change,status", [
    ({"requests": -1}, SHAPE), ({"tokens": -1}, SHAPE), ({"page_size": 12}, SHAPE),
    ({"max_pages": -1}, SHAPE), ({"num_free": -1}, SHAPE), ({"max_pages": 2 ** 28}, SHAPE),
    ({"requests": 2 ** 29, "max_pages": 4}, SHAPE), ({"tokens": 2 ** 30}, SHAPE),
    ({"context": None}, NULL), ({"new": None}, NULL), ({"free": None}, NULL),
    ({"table": None}, NULL), ({"cu": None}, NULL), ({"slots": None}, NULL),
    ({"positions": None}, NULL), ({"new_head": None}, NULL), ({"slots": FAKE + 4}, ALIGN),
    ({"context": FAKE + 2}, ALIGN), ({"head": FAKE + 1}, ALIGN),
    ({"head": FAKE, "new_head": FAKE}, SHAPE),
])
def test_cache_tables_rejects_before_launch(lib, change, status):
    assert _tables(lib, **change) == status


# ---------------------------------------------------------------- binding

def test_binding_refuses_before_launch(lib):
    q = torch.zeros(1, 4, 10, 32)
    with pytest.raises(ValueError, match="GPU"):
        na.sink_forward(q, q, q, 3)
    with pytest.raises(ValueError, match="batch, heads"):
        na.sink_forward(q[0], q[0], q[0], 3)
    with pytest.raises(ValueError, match="share batch"):
        na.sink_forward(q, q[:, :, :5], q[:, :, :5], 3)
    with pytest.raises(ValueError, match="multiple"):
        na.sink_forward(q, q[:, :3], q[:, :3], 3)
    with pytest.raises(TypeError, match="dtype"):
        na.sink_forward(q.double(), q.double(), q.double(), 3)
    with pytest.raises(TypeError, match="dtype"):
        na.sink_forward(q, q.half(), q.half(), 3)
    with pytest.raises(ValueError, match="last axis"):
        na.sink_forward(q.transpose(2, 3), q.transpose(2, 3), q.transpose(2, 3), 3)
    for f, name, least in ((lambda: sequence._count(0, "kernel_size", 1), "kernel_size", 1),
                           (lambda: sequence._count(-1, "sinks", 0), "sinks", 0)):
        with pytest.raises(ValueError, match=f"{name} must be at least {least}"):
            f()


def test_plans_are_looked_up_by_numbers(lib):
    # a tensor's value counts, not its identity; numbers that are not whole are refused
    w = torch.tensor(5)
    assert sequence._window(w, 2, torch.tensor(0.5)) == (5, 2, 0.5)
    w += 1
    assert sequence._window(w, 2, None) == (6, 2, None)
    with pytest.raises(TypeError):
        sequence._window(5.0, 2, None)
    with pytest.raises(TypeError):
        sequence._bounds(None, 100.5)
    # a growing bound: never below itself, at most a tile or 1/32 above, few distinct ones
    assert sequence._bounds(3, None) == (3, None)
    assert sequence._bounds(None, 0)[1] == 0 and sequence._bounds(None, -4)[1] == -4
    got = [sequence._bounds(None, n)[1] for n in range(1, 20000)]
    assert all(n <= x <= max(n + 31, n + n // 32) for n, x in enumerate(got, 1))
    assert len(set(got)) < 300


def test_cache_binding_refuses_before_launch(lib):
    pages = torch.zeros(4, 2, 16, 32)
    q, k = torch.zeros(3, 4, 32), torch.zeros(3, 2, 32)
    i32 = torch.zeros(2, dtype=torch.int32)
    table, cu = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    slots = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        na.cache_attention(q, pages, pages, table, i32, cu)
    with pytest.raises(ValueError, match="expected q"):
        na.cache_attention(q[0], pages, pages, table, i32, cu)
    with pytest.raises(ValueError, match="pages must be"):
        na.cache_attention(q, pages, pages[:3], table, i32, cu)
    with pytest.raises(ValueError, match="contiguous"):
        na.cache_attention(q, pages.transpose(1, 2), pages.transpose(1, 2), table, i32, cu)
    with pytest.raises(ValueError, match="GPU"):
        na.cache_write(k, k, slots, pages, pages)
    with pytest.raises(ValueError, match="expected k and v"):
        na.cache_write(k, k[:2], slots, pages, pages)
    with pytest.raises(ValueError, match="GPU"):
        na.cache_tables(i32, i32, table, i32, 16, 3)
    with pytest.raises(ValueError, match="one entry per request"):
        na.cache_tables(i32, i32[:1], table, i32, 16, 3)
    with pytest.raises(ValueError, match="max_pages"):
        na.cache_tables(i32, i32, table[:1], i32, 16, 3)
    with pytest.raises(ValueError, match="same new tokens"):
        na.cache_step(q, k[:2], k[:2], pages, pages, table, i32, i32, i32)


# ---------------------------------------------------------------- the plain forms

def test_visible_by_hand():
    i = torch.arange(6)
    seen = plain.visible(i, i, 2, 1).int().tolist()
    assert seen == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0],
                    [1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]


def test_plain_sink_is_the_softmax_of_the_visible_scores():
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(1, h, 9, 32, generator=gen) for h in (4, 2, 2))
    out, lse, _, _ = plain.sink(q, k, v, 3, 2, 0.2, lengths=[7])
    for h in range(4):
        for i in range(9):
            js = [j for j in range(min(i + 1, 7)) if i - j < 3 or j < 2] if i < 7 else []
            if not js:
                assert not bool(out[0, h, i].any()) and lse[0, h, i] == -math.inf
                continue
            s = torch.stack([(q[0, h, i].double() * k[0, h // 2, j].double()).sum() * 0.2 for j in js])
            w = torch.exp(s) / torch.exp(s).sum()
            ref = sum(a * v[0, h // 2, j].double() for a, j in zip(w, js))
            assert float((out[0, h, i] - ref).abs().max()) < 1e-12
            assert abs(float(lse[0, h, i] - torch.exp(s).sum().log())) < 1e-12


@pytest.mark.parametrize("W,S,lengths", [(3, 2, None), (1, 0, None), (100, 0, [7]), (2, 5, [9])])
def test_plain_gradient_is_that_of_the_plain_forward(W, S, lengths):
    gen = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(1, h, 9, 32, generator=gen).double() for h in (4, 2, 2))
    dout = torch.randn(1, 4, 9, 32, generator=gen).double()
    scale = 0.3

    # (plain.sink takes its bounds from a type: fp32 stands in, the values stay 64-bit)
    def loss(q, k, v):
        n = 9 if lengths is None else lengths[0]
        pos = torch.arange(n)
        seen = plain.visible(pos, pos, W, S)
        total = 0.0
        for h in range(4):
            r = plain.attend(q[0, h, :n], k[0, h // 2, :n], v[0, h // 2, :n], seen, scale,
                             torch.float32)
            total += float((r[0] * dout[0, h, :n]).sum())
        return total

    out, lse = torch.zeros_like(q), torch.full((1, 4, 9), -math.inf).double()
    n = 9 if lengths is None else lengths[0]
    pos = torch.arange(n)
    for h in range(4):
        r = plain.attend(q[0, h, :n], k[0, h // 2, :n], v[0, h // 2, :n],
                         plain.visible(pos, pos, W, S), scale, torch.float32)
        out[0, h, :n], lse[0, h, :n] = r[:2]
    plain.HALF[torch.float64] = 0.0
    grads, _ = plain.sink_grad(q, k, v, out, lse, dout, W, S, scale, lengths)
    del plain.HALF[torch.float64]
    step = 1e-5
    for i, g in enumerate(grads):  # central differences along random directions
        for _ in range(3):
            d = torch.randn(g.shape, generator=gen).double()
            x = [q, k, v]
            up, down = list(x), list(x)
            up[i], down[i] = x[i] + step * d, x[i] - step * d
            slope = (loss(*up) - loss(*down)) / (2 * step)
            assert abs(slope - float((g * d).sum())) < 1e-7 * (1 + abs(slope))


def test_plain_tables_by_hand():
    table = [[5, -1, -1], [-1, -1, -1]]
    got = plain.tables([15, 0], [2, 17], table, [8, 3, 9], 16, 20)
    assert got == ([0, 2, 19], [95, 128] + list(range(48, 64)) + [144, -1],
                   [15, 16] + list(range(17)) + [-1], 3)
    assert table == [[5, 8, -1], [3, 9, -1]]


def test_plain_cache_is_plain_sink_over_the_pages():
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(1, h, 40, 32, generator=gen) for h in (2, 1, 1))
    ids = [2, 0, 1]
    kp, vp = torch.zeros(3, 1, 16, 32), torch.zeros(3, 1, 16, 32)
    for t in range(40):
        kp[ids[t // 16], :, t % 16], vp[ids[t // 16], :, t % 16] = k[0, :, t], v[0, :, t]
    want = plain.sink(q, k, v, 10, 3, 0.3)
    got = plain.cache(q[0, :, 25:].transpose(0, 1), kp, vp, [ids], [25], [15], 10, 3, 0.3)
    assert float((got[0].transpose(0, 1) - want[0][0, :, 25:]).abs().max()) < 1e-12
    assert float((got[1].T - want[1][0, :, 25:]).abs().max()) < 1e-12
