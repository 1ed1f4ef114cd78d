"""What a chunk store does when a call is refused under way, and where requests lie side by side (buffers on the host; calls are recorded, none runs)."""
import pytest
import torch

from paper_2609_33503_b200 import binding as B
from paper_2609_33503_b200.chunk_store import ChunkStore
from tests.test_continuations_binding import bf
from tests.test_continuations_class_host import D, HKV, L, caches
from tests.test_quantized_paths_host import chunk_store


@pytest.mark.parametrize("layer", range(L))
def test_blocks_of_a_chunk_that_is_refused_stay_free(monkeypatch, layer):
    """An append that raises, at any layer: no chunk, no block less, and the next one is put where it would have been."""
    s, calls = chunk_store(monkeypatch)
    s.put("a", caches(), 0, 0, 20, 0)
    free, append, seen = list(s.free), B.relaxkv_append_quantized, []

    def failing(*a, **kw):
        seen.append(1)
        if len(seen) > layer:
            raise RuntimeError("the append failed")
        return append(*a, **kw)

    monkeypatch.setattr(B, "relaxkv_append_quantized", failing)
    for _ in range(3):
        seen.clear()
        with pytest.raises(RuntimeError, match="append failed"):
            s.put("b", caches(), 0, 20, 40, 20)
        assert s.free == free and "b" not in s
    monkeypatch.setattr(B, "relaxkv_append_quantized", append)
    s.put("b", caches(), 0, 20, 40, 20)
    assert s.chunks["b"].slots.tolist() == list(range(32, 72)) and len(s.free) == len(free) - 3


def test_a_cache_that_the_library_refuses_costs_no_blocks(monkeypatch):
    """Rows of another type than the store takes: refused by the binding, before any call."""
    s, calls = chunk_store(monkeypatch)
    odd = [B.CacheView(bf(70, HKV, D), bf(70, HKV, D), [0]) for _ in range(L)]
    for c in odd:
        c.k, c.v = c.k.half(), c.v.half()
    with pytest.raises(ValueError):
        s.put("a", odd, 0, 0, 20, 0)
    assert not calls and len(s.free) == 10 and "a" not in s


def test_a_request_ends_where_the_next_one_begins(monkeypatch):
    """Three requests in one cache, in any order: chunks are neither put together over the next one's tokens nor kept with them."""
    s, calls = chunk_store(monkeypatch, n_blocks=20)
    s.put("a", caches(), 0, 0, 30, 0)
    s.put("b", caches(), 0, 30, 20, 30)
    view = lambda: [B.CacheView(bf(140, HKV, D), bf(140, HKV, D), [60, 0, 100]) for _ in range(L)]        # 40, 60 and 40 tokens
    calls.clear()
    for req, keys, first in ((0, ["a", "b"], 0), (0, ["a"], 11), (1, ["a", "b"], 11), (2, ["a", "b"], 0), (2, ["b"], 21)):
        with pytest.raises(ValueError, match="tokens"):
            s.assemble(keys, view(), req, first)
    for req, first, n in ((0, 0, 41), (0, 30, 11), (1, 50, 11), (2, 0, 41)):
        with pytest.raises(ValueError, match="tokens"):
            s.put("c", view(), req, first, n, 0)
    assert not calls and "c" not in s
    assert s.assemble(["a"], view(), 0, 10) == 30 and s.assemble(["a", "b"], view(), 1, 10) == 50 and s.assemble(["b", "b"], view(), 2) == 40
    s.put("c", view(), 1, 0, 60, 0)
    # layers that do not agree on it: the shorter one holds
    mixed = view()
    mixed[1] = B.CacheView(bf(140, HKV, D), bf(140, HKV, D), [60, 0, 80])
    with pytest.raises(ValueError, match="tokens"):
        s.assemble(["a"], mixed, 0)


def test_requests_that_share_their_first_token(monkeypatch):
    """Two views of the same tokens: each reaches to where another one begins."""
    view = B.CacheView(bf(50, HKV, D), bf(50, HKV, D), [0, 0, 20])
    assert [view.tokens(b) for b in range(3)] == [20, 20, 30]
    assert B.CacheView(bf(50, HKV, D), None, [60]).tokens(0) == 0
