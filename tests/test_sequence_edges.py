"""Edges of the sequence operators that need no GPU: refusals, and first use by several threads."""
import pytest
import torch

import paper_2403_04690_amd as na
from paper_2403_04690_amd import sequence
from tests import test_sequence_host as host

SHAPE, NULL = host.SHAPE, host.NULL
lib = host.lib  # (a fixture)


# ---------------------------------------------------------------- no query heads

def test_key_heads_without_query_heads_are_refused(lib):
    """Gradients of keys that no query head reads would be left unwritten."""
    p = host._sink(heads=0, kv_heads=2)
    assert host._forward(lib, p) == SHAPE and host._backward(lib, p) == SHAPE
    assert lib.na_sink_backward_workspace(p) == 0
    assert host._attend(lib, host._cache(heads=0, kv_heads=2)) == SHAPE
    q, k = torch.zeros(1, 0, 5, 32), torch.zeros(1, 2, 5, 32)
    lse = torch.zeros(1, 0, 5)
    with pytest.raises(ValueError, match="multiple"):
        na.sink_forward(q, k, k, 3)
    with pytest.raises(ValueError, match="multiple"):
        na.sink_backward(q, k, k, q, lse, q, 3)
    with pytest.raises(ValueError, match="multiple"):
        na.sink_attention(q, k.requires_grad_(True), k, 3)
    pages, ints = torch.zeros(4, 2, 16, 32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="multiple"):
        na.cache_attention(torch.zeros(3, 0, 32), pages, pages, torch.zeros(2, 3, dtype=torch.int32),
                           ints, torch.zeros(3, dtype=torch.int32))


# ---------------------------------------------------------------- axes of one entry

@pytest.mark.parametrize("size,stride", [
    ({"batch": 1}, lambda b, h, t: (3, h, t)), ({"batch": 1}, lambda b, h, t: (-8, h, t)),
    ({"tokens": 1}, lambda b, h, t: (b, h, 2 ** 40)), ({"heads": 2, "kv_heads": 1}, None),
    ({"heads": 1, "kv_heads": 1}, lambda b, h, t: (b, 5, t)),
])
def test_strides_of_axes_of_one_entry_are_not_looked_at(lib, size, stride):
    p = host._sink(**size)
    for name in host.STRIDED:
        s = getattr(p, name)
        if stride is not None:
            setattr(p, name, sequence._Strides(*stride(s.batch, s.head, s.token)))
        elif name in ("k", "v", "dk", "dv"):
            s.head = 7
    # (a valid problem: the pointer is what is refused)
    assert host._forward(lib, p, q=None) == NULL and host._backward(lib, p, q=None) == NULL
    assert lib.na_sink_backward_workspace(p) > 0


def test_cache_strides_of_axes_of_one_entry_are_not_looked_at(lib):
    for size, odd in (({"tokens": 1}, (0, 64, 2 ** 40 + 1)),
                      ({"heads": 1, "kv_heads": 1}, (0, 3, 64))):
        p = host._cache(q=odd, k=odd, v=odd, out=odd, **size)
        assert host._attend(lib, p, q=None) == NULL and host._write(lib, p, k=None) == NULL


# ---------------------------------------------------------------- first use

def test_first_use_by_many_threads_while_the_extension_is_imported(lib, monkeypatch):
    """A thread that comes while another one binds the library finds every entry point."""
    import builtins
    import threading
    import time

    names = {"na_sink_forward", "na_sink_backward", "na_cache_tables", "na_cache_write",
             "na_cache_attention"}
    monkeypatch.setattr(sequence, "_bound", None)
    monkeypatch.setattr(sequence, "_entry", {})
    real = builtins.__import__

    def slow(name, *args, **kwargs):
        if name.endswith("_na_fast"):
            time.sleep(0.2)
        return real(name, *args, **kwargs)

    monkeypatch.setattr(builtins, "__import__", slow)
    wrong = []

    def use():
        sequence._library()
        wrong.extend(names - set(sequence._entry))

    threads = [threading.Thread(target=use) for _ in range(8)]
    for t in threads:
        t.start()
        time.sleep(0.01)
    for t in threads:
        t.join(20)
    assert wrong == []
