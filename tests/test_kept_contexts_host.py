"""Steps over contexts that are kept in 8 bits: rows of a sequence whose context is not in the store are refused (buffers on the host; the calls that would be made
are recorded, none runs)."""
import pytest
import torch

from paper_2609_33503_b200 import binding as B
from paper_2609_33503_b200.continuations import Continuations
from tests.test_continuations_binding import Recorder, bf
from tests.test_continuations_class_host import BLK, D, H, HKV, L, caches


def make(monkeypatch, ctx=(70,), seqs=(3,), **kw):
    monkeypatch.undo()
    c = Continuations(H, HKV, D, ctx, seqs, L, BLK, **dict(dict(n_blocks=40, max_len=40, block_size=16, max_rows=32, device="cpu", store_dtype=torch.int8), **kw))
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    return c, r.calls


def test_no_rows_before_their_context(monkeypatch):
    c, calls = make(monkeypatch)
    for new in ([1, 0, 0], [1, 1, 1], [0, 0, 5], [-1, 1, 0]):
        with pytest.raises(ValueError, match="not in the store"):
            c.begin(new)
    assert not calls and c.lens == [0, 0, 0] and c.n_free == 40
    assert c.begin([0, 0, 0]) == 0                       # who waits needs none
    c.keep_contexts(caches(), [0, 2])
    assert c.begin([1, 0, 2]) == 3 and c.lens == [71, 0, 72]
    with pytest.raises(ValueError, match=r"\[1\]"):
        c.begin([1, 1, 1])


def test_a_context_goes_with_its_sequence(monkeypatch):
    """Ended and begun again: with its context kept again, not without."""
    c, calls = make(monkeypatch)
    c.keep_contexts(caches())
    c.begin([2, 1, 1])
    c.begin([1, -1, 0])
    n = len(calls)
    with pytest.raises(ValueError, match=r"\[1\]"):
        c.begin([0, 3, 0])
    assert len(calls) == n and c.lens == [73, 0, 71]
    c.keep_contexts(caches(), [1])
    assert c.begin([0, 3, 0]) == 3 and c.lens == [73, 73, 71]


def test_a_context_that_is_kept_in_part_is_not_there(monkeypatch):
    """An append that fails in the second step of a context: its rows stay refused until it has been kept whole."""
    c, calls = make(monkeypatch, seqs=(1,), max_rows=50)
    append, seen = B.relaxkv_append_quantized, []

    def failing(*a, **kw):
        seen.append(1)
        if len(seen) > L:
            raise RuntimeError("the append failed")
        return append(*a, **kw)

    monkeypatch.setattr(B, "relaxkv_append_quantized", failing)
    with pytest.raises(RuntimeError, match="append failed"):
        c.keep_contexts(caches())
    with pytest.raises(ValueError, match="not in the store"):
        c.begin([1])
    monkeypatch.setattr(B, "relaxkv_append_quantized", append)
    c.begin([-1])
    c.keep_contexts(caches())
    assert c.begin([1]) == 1 and c.lens == [71]


def test_sequences_without_a_context_and_stores_of_bf16_need_none(monkeypatch):
    c, _ = make(monkeypatch, ctx=(0, 70), seqs=(2, 1))
    assert c.begin([1, 2, 0]) == 3 and c.begin([-1, 1, 0]) == 1 and c.begin([4, 0, -1]) == 4
    with pytest.raises(ValueError, match=r"\[2\]"):
        c.begin([1, 1, 1])
    c, _ = make(monkeypatch, store_dtype=None)
    assert c.begin([1, 1, 1]) == 3 and c.begin([-1, 1, 1]) == 2 and c.begin([5, 0, 0]) == 5


def test_a_refused_step_changes_nothing(monkeypatch):
    """A step that ends a sequence and is refused for its size: the sequence's context is still there."""
    c, calls = make(monkeypatch)
    c.keep_contexts(caches())
    with pytest.raises(ValueError, match="rows"):
        c.begin([-1, 33, 0])
    assert c.begin([1, 0, 0]) == 1 and c.lens == [71, 70, 70]
