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
