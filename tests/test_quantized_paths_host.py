"""What the classes over contexts in 8 bits ask for and refuse (buffers on the host; the calls that would be made are recorded, none runs)."""
import pytest
import torch

from paper_2609_33503_b200 import binding as B
from paper_2609_33503_b200 import inputs
from paper_2609_33503_b200.chunk_store import ChunkStore
from paper_2609_33503_b200.continuations import Continuations
from paper_2609_33503_b200.query_pass import QueryPass
from tests.test_continuations_binding import Recorder, bf
from tests.test_continuations_class_host import BLK, D, H, HKV, L, caches, weights


def record(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    return r.calls


def rotary(dims=D):
    return B.Rotary.scaled(dims, 1e4, device="cpu")


def make(monkeypatch, ctx=(70,), seqs=(3,), **kw):
    monkeypatch.undo()
    kw = dict(dict(n_blocks=20, max_len=40, block_size=16, max_rows=32, device="cpu", store_dtype=torch.int8), **kw)
    c = Continuations(H, HKV, D, ctx, seqs, L, BLK, **kw)
    return c, record(monkeypatch)


def names(calls):
    return [name for name, _ in calls]


@pytest.mark.parametrize("kw", [dict(n_select=2), dict(store_dtype=torch.bfloat16), dict(store_dtype=torch.uint8)])
def test_what_a_store_is_not_made_for(monkeypatch, kw):
    with pytest.raises(ValueError):
        make(monkeypatch, **kw)


def test_contexts_are_kept_in_steps_of_the_rooms_size(monkeypatch):
    c, calls = make(monkeypatch, ctx=(70, 0, 9), seqs=(1, 1, 2))
    room = [B.CacheView(bf(100, HKV, D), bf(100, HKV, D), [3, 80, 80]) for _ in range(L)]
    c.keep_contexts(room)
    assert c.lens == [70, 0, 9, 9] and c.n_rows == 0 and c.n_free == 20 - 5 - 2
    appends = [a for name, a in calls if name == "relaxkv_append_quantized"]
    rows = [(a[9], (a[5] - room[0].k.data_ptr()) // (2 * HKV * D)) for a in appends if room[0].k.data_ptr() <= a[5] < room[0].k.data_ptr() + room[0].k.nbytes]
    assert rows == [(32, 3), (32, 35), (6, 67), (9, 80), (9, 80)] and len(appends) == L * 5
    assert names(calls).count("relaxkv_build_block_tables") == 3
    assert all(a[1] is None for a in appends)                                    # no queries



def test_a_step_runs_over_the_store_alone(monkeypatch):
    c, calls = make(monkeypatch)
    c.keep_contexts(caches())
    calls.clear()
    assert c.begin([2, 1, 0]) == 3
    assert c.run(bf(3, 256), weights()).shape == (3, 256)
    n = names(calls)
    assert n.count("relaxkv_append_quantized") == n.count("relaxkv_quantized_attention") == L
    assert not [x for x in n if "paged" in x or "prefix" in x or "rope" in x]
    assert c.rows.c.max_len == 72 and c.width * 16 >= 70 + 40
    with pytest.raises(ValueError):
        c.attention(0, None, bf(4, H, D), bf(4, H, D))


def test_contexts_that_cannot_be_kept(monkeypatch):
    c, calls = make(monkeypatch)
    c.keep_contexts(caches())
    before = len(calls)
    for bad in (lambda: c.keep_contexts(caches()), lambda: c.keep_contexts(caches(), [3]), lambda: c.keep_contexts(caches(), [-1])):
        with pytest.raises(ValueError):
            bad()
    assert len(calls) == before
    c.begin([0, -1, 0])
    with pytest.raises(ValueError):
        c.keep_contexts(caches()[:1], [1])
    with pytest.raises(ValueError):
        c.keep_contexts([None] * L, [1])
    with pytest.raises(ValueError):
        c.keep_contexts([B.CacheView(bf(69, HKV, D), bf(69, HKV, D), [0])] * L, [1])
    with pytest.raises(ValueError):
        c.keep_contexts([B.CacheView(bf(70, HKV, 2 * D), bf(70, HKV, 2 * D), [0])] * L, [1])
    assert c.lens == [70, 0, 70]
    c.keep_contexts(caches(), [1])
    assert c.lens == [70, 70, 70]
    small, calls = make(monkeypatch, n_blocks=14)
    with pytest.raises(ValueError, match="1 blocks short"):
        small.keep_contexts(caches())
    assert not calls and small.lens == [0, 0, 0]
    monkeypatch.undo()
    plain = Continuations(H, HKV, D, (70,), (1,), L, BLK, n_blocks=9, max_len=40, block_size=16, device="cpu")
    with pytest.raises(ValueError):
        plain.keep_contexts(caches())
    record(monkeypatch)
    plain.begin([1])
    with pytest.raises(ValueError):
        plain.run(bf(1, 256), weights())


def test_no_context_needs_no_caches(monkeypatch):
    c, calls = make(monkeypatch, ctx=(0,), seqs=(2,))
    c.keep_contexts([])
    assert not calls and c.begin([1, 1]) == 2


@pytest.mark.parametrize("scaled", [False, True])
def test_a_models_rotary_takes_the_place_of_its_theta(monkeypatch, scaled):
    blk = inputs.BlockShape(hidden=256, inter=384, rotary=rotary(32) if scaled else None)
    qp = QueryPass(H, HKV, D, (40,), (5,), blk, device="cpu")
    c = Continuations(H, HKV, D, (40,), (1,), L, blk, n_blocks=9, max_len=40, block_size=16, max_rows=4, device="cpu")
    calls = record(monkeypatch)
    room = [B.CacheView(bf(50, HKV, D), bf(50, HKV, D), [0]) for _ in range(L)]
    qp.prefill(bf(5, 256), weights(), room)
    n = names(calls)
    assert n.count("relaxkv_qk_norm_rotate") == n.count("relaxkv_scatter_kv_lists") == L * scaled and n.count("relaxkv_qk_norm_rope_append") == L * (not scaled)
    calls.clear()
    c.begin([3])
    c.run(bf(3, 256), weights(), room)
    n = names(calls)
    assert n.count("relaxkv_qk_norm_rotate") == L * scaled and n.count("relaxkv_qk_norm_rope_append_paged") == L


def chunk_store(monkeypatch, n_blocks=10):
    s = ChunkStore(L, HKV, D, n_blocks, rotary(), block_size=16, device="cpu")
    return s, record(monkeypatch)


def test_chunks_take_blocks_and_give_them_back(monkeypatch):
    s, calls = chunk_store(monkeypatch)
    s.put("a", caches(), 0, 0, 40, 0)
    s.put("b", caches(), 0, 40, 16, 40)
    assert names(calls) == ["relaxkv_append_quantized"] * 2 * L and len(s.free) == 6 and s.tokens("a") == 40 and "b" in s and "c" not in s
    assert s.chunks["a"].slots.tolist() == list(range(40)) and s.chunks["b"].slots.tolist() == list(range(48, 64))
    s.drop("a")
    assert len(s.free) == 9 and "a" not in s
    s.put("c", caches(), 0, 0, 70, 0)
    assert sorted(s.chunks["c"].blocks + s.chunks["b"].blocks + tuple(s.free)) == list(range(10))
    with pytest.raises(KeyError):
        s.drop("a")


def test_a_context_is_put_together_in_one_call_per_layer(monkeypatch):
    s, calls = chunk_store(monkeypatch)
    s.put("a", caches(), 0, 0, 20, 0)
    s.put("b", caches(), 0, 20, 10, 20)
    calls.clear()
    room = [B.CacheView(bf(70, HKV, D), bf(70, HKV, D), [4]) for _ in range(L)]
    assert s.assemble(["b", "a", "b"], room, 0, 2) == 40
    assert names(calls) == ["relaxkv_read_quantized"] * L and all(a[2] == 40 and a[5] is not None and a[6] is not None for _, a in calls)
    assert calls[0][1][7] == room[0].k.data_ptr() + 6 * HKV * D * 2
    calls.clear()
    assert s.assemble(["a", "b"], room) == 30                # where they were: nothing to turn
    assert all(a[5] is None and a[6] is None for _, a in calls)
    calls.clear()
    assert s.assemble([], room) == 0 and not calls


def test_keys_that_are_turned_on_do_not_grow_again():
    yarn = B.Rotary.scaled(D, 1e4, "ramp", 8.0, 4096, 1.0, 32.0, device="cpu")
    assert yarn.amplitude > 1.2 and ChunkStore(1, HKV, D, 2, yarn, block_size=16, device="cpu").turn.amplitude == 1.0


@pytest.mark.parametrize("bad", [
    lambda s, c: s.put("a", c, 0, 0, 8, 0), lambda s, c: s.put("n", c, 0, 0, 0, 0), lambda s, c: s.put("n", c, 0, 60, 11, 0), lambda s, c: s.put("n", c, 0, -1, 8, 0),
    lambda s, c: s.put("n", c, 1, 0, 8, 0), lambda s, c: s.put("n", c[:1], 0, 0, 8, 0), lambda s, c: s.assemble(["a"], c, 0, 55), lambda s, c: s.assemble(["a"], c[:1]),
    lambda s, c: s.assemble(["a"], c, -1), lambda s, c: s.put("n", [B.CacheView(bf(70, HKV, D), None, [0])] * L, 0, 0, 8, 0),
    lambda s, c: s.put("n", [B.CacheView(bf(70, HKV, 2 * D), bf(70, HKV, 2 * D), [0])] * L, 0, 0, 8, 0)],
    ids=["twice", "empty", "beyond", "before", "request", "layers", "assembled beyond", "assembled layers", "assembled request", "no values", "dims"])
def test_what_a_chunk_store_refuses(monkeypatch, bad):
    s, calls = chunk_store(monkeypatch)
    s.put("a", caches(), 0, 0, 20, 0)
    n, free = len(calls), list(s.free)
    with pytest.raises(ValueError):
        bad(s, caches())
    assert len(calls) == n and s.free == free


def test_a_full_chunk_store_says_so(monkeypatch):
    s, calls = chunk_store(monkeypatch, n_blocks=3)
    s.put("a", caches(), 0, 0, 20, 0)
    with pytest.raises(ValueError, match="1 blocks short"):
        s.put("b", caches(), 0, 0, 17, 0)
    with pytest.raises(KeyError):
        s.assemble(["b"], caches())
    assert len(s.free) == 1


def test_rows_of_heads_as_the_calls_take_them():
    x = bf(6, 4, 64)
    assert B._head_rows(x, None, None, None, None) == B._head_rows(x, bf(6, 4, 64), 6, 4, 64) == B._head_rows(x, x, 6, None, None) == (6, 4, 64, 256, 64)
    assert B._head_rows(x.transpose(0, 1), None, 4, 6, 64) == (4, 6, 64, 64, 256)
    assert B._head_rows(x[:, :, :32], x[:, :, 32:], None, None, 32) == (6, 4, 32, 256, 64)
    # the distance to a row or head that is not there: at least a head's dims
    assert B._head_rows(torch.as_strided(x, (1, 1, 64), (0, 0, 1)), None, None, None, None) == (1, 1, 64, 64, 64)
    assert B._head_rows(torch.as_strided(x, (1, 2, 64), (3, 64, 1)), None, None, None, None) == (1, 2, 64, 64, 64)
    assert B._head_rows(x[:0], x[:0], 0, 4, 64) == (0, 4, 64, 256, 64)


@pytest.mark.parametrize("args", [
    (bf(6, 4, 64).float(), None, None, None, None), (bf(6, 4, 64).half(), None, None, None, None), (bf(6, 256), None, None, None, None), (bf(6, 4, 2, 64), None, None, None, None),
    (bf(6, 4, 128)[..., ::2], None, None, None, None), (bf(6, 4, 64), None, 5, None, None), (bf(6, 4, 64), None, None, 3, None), (bf(6, 4, 64), None, None, None, 128),
    (bf(6, 4, 64), bf(6, 4, 64).float(), None, None, None), (bf(6, 4, 64), bf(6, 2, 64), None, None, None), (bf(6, 4, 64), bf(4, 6, 64).transpose(0, 1), None, None, None),
    (bf(6, 4, 64), bf(6, 256), None, None, None)])
def test_rows_of_heads_that_are_refused(args):
    with pytest.raises(ValueError, match="rows"):
        B._head_rows(*args)


def test_rows_of_heads_keep_no_reference():
    import sys
    x, y = bf(2, 2, 64), bf(2, 2, 64)
    B._head_rows(x, y, None, None, None)
    before = [sys.getrefcount(o) for o in (x, y, torch.bfloat16)]
    for _ in range(200):
        B._head_rows(x, y, 2, 2, 64)
        with pytest.raises(ValueError):
            B._head_rows(x, y, 3, 2, 64)
    assert [sys.getrefcount(o) for o in (x, y, torch.bfloat16)] == before
    for bad in ((3, None, None, None, None), (x, 3, None, None, None)):
        with pytest.raises(AttributeError):
            B._head_rows(*bad)
    with pytest.raises(TypeError):
        B._head_rows(x, None, "a", None, None)
