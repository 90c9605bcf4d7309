"""The decoder example's page bookkeeping (host only)."""
import pytest
import torch

from paper_2502_06786_b200 import serve


def _cache(pages=6):
    return serve.PagedCache(serve.Config(layers=1, kv_heads=1, head_dim=64, page_size=16), pages, device="cpu")


def _state(c):
    return {s: list(p) for s, p in c.pages.items()}, dict(c.length), list(c.free)


def test_a_batch_that_does_not_fit_changes_nothing():
    c = _cache()
    serve.Batch(c, [("a", 20), ("b", 3)], device="cpu")
    before = _state(c)
    for steps in ([("a", 1), ("c", 100)], [("c", 40), ("d", 40)], [("b", 14), ("a", 60)]):
        with pytest.raises(RuntimeError, match="full"):
            serve.Batch(c, steps, device="cpu")
        assert _state(c) == before
    with pytest.raises(KeyError):
        c.release("c")                                          # never came to be
    c.release("a")
    c.release("b")
    assert sorted(c.free) == list(range(6)) and not c.pages and not c.length


def test_a_refused_sequence_leaves_no_trace():
    c = _cache(2)
    c.extend("a", 32)
    with pytest.raises(RuntimeError, match="full"):
        c.extend("b", 1)
    assert "b" not in c.pages and "b" not in c.length
    with pytest.raises(RuntimeError, match="full"):
        c.extend("a", 1)
    assert c.length["a"] == 32 and len(c.pages["a"]) == 2


def test_batch_arrays():
    c = _cache()
    b = serve.Batch(c, [("a", 20), ("b", 3)], device="cpu")
    assert b.cu_q.tolist() == [0, 20, 23] and b.kv_len.tolist() == [20, 3] and (b.max_q, b.max_kv) == (20, 20)
    assert b.page_table.tolist() == [c.pages["a"], c.pages["b"] + [-1]]
    b = serve.Batch(c, [("b", 14), ("a", 1)], device="cpu")
    assert b.kv_len.tolist() == [17, 21] and len(c.pages["b"]) == 2 and len(c.pages["a"]) == 2
    with pytest.raises(ValueError):
        serve.Batch(c, [("a", 1), ("a", 1)], device="cpu")


def test_positions_past_the_rotation_table_are_refused_before_anything_runs():
    model = serve.Decoder.__new__(serve.Decoder)                # no weights: refused before they are needed
    model.cfg, model.layers, model.cos_sin = serve.Config(max_pos=30), [], None
    c = _cache()
    x = torch.zeros(30, 512, dtype=torch.bfloat16)
    assert model.forward(x, c, serve.Batch(c, [("a", 30)], device="cpu")).shape == (30, 512)
    with pytest.raises(ValueError, match="30 positions"):
        model.forward(x[:1], c, serve.Batch(c, [("a", 1)], device="cpu"))
