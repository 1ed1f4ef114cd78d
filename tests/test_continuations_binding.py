"""Tensors that are too small, of another type or out of order for a call over continuations are refused before the call (host tensors; the
calls that would be made are recorded, none runs)."""
import pytest
import torch

from paper_2609_33503_b200 import binding as B


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or B.OK


@pytest.fixture
def calls(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    return r.calls


def i32(*n):
    return torch.zeros(*n, dtype=torch.int32)


def bf(*n):
    return torch.zeros(*n, dtype=torch.bfloat16)


def tables(**kw):
    n, rows = 6, 9
    a = dict(seq_len=i32(n), new_len=i32(n), seq_base=i32(n), free_blocks=i32(40), n_free=i32(1), block_table=i32(n, 5), seq_len_out=i32(n), n_free_out=i32(1),
             row_cu=i32(n + 1), row_seq=i32(rows), row_pos=i32(rows), row_len=i32(rows), row_slot=i32(rows))
    a.update(kw)
    return a


SHORT = dict(new_len=5, seq_base=5, n_free=0, seq_len_out=5, n_free_out=0, row_cu=6, row_pos=8, row_len=8, row_slot=8)


@pytest.mark.parametrize("name", list(SHORT))
def test_block_tables_refuse_short_tensors_and_other_types(calls, name):
    with pytest.raises(ValueError):
        B.relaxkv_build_block_tables(16, **tables(**{name: i32(SHORT[name])}), stream=0)
    with pytest.raises(ValueError):
        B.relaxkv_build_block_tables(16, **tables(**{name: torch.zeros(SHORT[name] + 1, dtype=torch.int64)}), stream=0)
    assert not calls


def test_block_tables_refuse_other_tables_and_orders(calls):
    for kw in (dict(block_table=i32(5, 5)), dict(block_table=torch.zeros(6, 5, dtype=torch.int64)), dict(new_len=i32(1).expand(6)), dict(new_len=i32(6, 2)[:, 0]),
               dict(seq_base=i32(1).expand(6)), dict(seq_len=torch.zeros(6, dtype=torch.int64)), dict(free_blocks=torch.zeros(40, dtype=torch.int16)),
               dict(row_seq=torch.zeros(9, dtype=torch.int64)), dict(row_slot=i32(12).expand(2, 12))):
        with pytest.raises(ValueError):
            B.relaxkv_build_block_tables(16, **tables(**kw), stream=0)
    assert not calls


def test_block_tables_take_what_they_took(calls):
    t = tables(seq_base=None, row_cu=i32(20), row_pos=i32(100), row_slot=B.Offsets(i32(30), 4), block_table=i32(8, 7)[1:, 2:])
    B.relaxkv_build_block_tables(16, **t, stream=0)
    name, a = calls[0]
    assert name == "relaxkv_build_block_tables" and len(a) == 20 and a[:2] == (6, 16) and a[4] is None
    assert a[2] == t["seq_len"].data_ptr() and a[6:8] == (40, t["n_free"].data_ptr()) and a[8:12] == (t["block_table"].data_ptr(), 5, 7, 9)
    assert a[12:19] == tuple(t[k].data_ptr() for k in ("seq_len_out", "n_free_out", "row_cu", "row_seq", "row_pos", "row_len", "row_slot"))
    B.relaxkv_build_block_tables(16, **tables(**{k: i32(0) for k in ("row_seq", "row_pos", "row_len", "row_slot")}), stream=0)
    assert calls[1][1][11] == 0


def append(**kw):
    n, H, Hkv, D = 5, 8, 2, 64
    a = dict(store=B.PagedStore(bf(4, 16, Hkv, D), bf(4, 16, Hkv, D)), q=bf(n, H, D), k=bf(n, Hkv, D), v=bf(n, Hkv, D), positions=i32(n), slots=i32(n), theta=1e4,
             q_out=bf(n, H, D))
    a.update(kw)
    return a


APPEND = [dict(store=B.PagedStore(bf(4, 16, 1, 64), bf(4, 16, 1, 64))), dict(store=B.PagedStore(bf(4, 16, 2, 128), bf(4, 16, 2, 128))),
          dict(store=B.PagedStore(bf(4, 16, 4, 32), bf(4, 16, 4, 32))), dict(k=bf(5, 3, 64)), dict(k=bf(4, 2, 64)), dict(v=bf(5, 1, 64)), dict(v=bf(4, 2, 64)),
          dict(q=bf(5, 12, 64)[:, :8]), dict(q=bf(5, 8, 64).float()), dict(k=bf(5, 12, 64)[:, 8:10]), dict(v=bf(5, 12, 64)[:, 10:]), dict(q_out=bf(4, 8, 64)),
          dict(positions=i32(4)), dict(slots=i32(4)), dict(slots=torch.zeros(5, dtype=torch.int64)), dict(positions=torch.zeros(5, dtype=torch.int64)),
          dict(w_q_norm=bf(32), w_k_norm=bf(64)), dict(w_q_norm=bf(64), w_k_norm=bf(64).float())]


@pytest.mark.parametrize("i", range(len(APPEND)))
def test_append_refuses_what_does_not_fit_the_rows_or_the_store(calls, i):
    with pytest.raises(ValueError):
        B.relaxkv_qk_norm_rope_append_paged(**append(**APPEND[i]), stream=0)
    assert not calls


def test_append_takes_what_it_took(calls):
    for kw in (dict(), dict(k=bf(9, 1, 64)), dict(w_q_norm=bf(64), w_k_norm=bf(64)), dict(slots=i32(9)), dict(q_out=bf(9, 8, 64))):
        a = append(**kw)
        B.relaxkv_qk_norm_rope_append_paged(**a, stream=0)
        got = calls[-1][1]
        assert got[1:8] == (a["q"].data_ptr(), a["k"].data_ptr(), a["v"].data_ptr(), 5, 8, a["k"].shape[1], 64) and len(got) == 16
        assert got[11:13] == (a["positions"].data_ptr(), a["slots"].data_ptr()) and got[14] == a["q_out"].data_ptr()


def step(n_rows=7, H=8, Hkv=2, D=64, ctx=(100, 0, 33), seqs=(2, 1, 2)):
    """What the attention calls take, by name."""
    cu = [sum(seqs[:i]) for i in range(len(seqs) + 1)]
    shape = B.Shape(H, Hkv, D, ctx)
    at = [sum(ctx[:i]) for i in range(len(ctx))]
    nb = sum(-(-t // 16) for t in ctx)
    rows = B.ContinuationRows(cu, [n_rows] * len(ctx), 40, i32(cu[-1] + 1), i32(n_rows), i32(n_rows), i32(cu[-1], 3))
    return dict(shape=shape, cache=B.CacheView(bf(sum(ctx), Hkv, D), bf(sum(ctx), Hkv, D), at), store=B.PagedStore(bf(9, 16, Hkv, D), bf(9, 16, Hkv, D)), rows=rows,
                q=bf(n_rows, H, D), out=bf(n_rows, H, D), lse_out=torch.zeros(H, n_rows), blocks=i32(n_rows, Hkv, 4), bounds=torch.zeros(nb, Hkv, 2, D, dtype=torch.int8),
                scale=torch.zeros(nb, Hkv), workspace=torch.zeros(512, dtype=torch.uint8))


def shared(a):
    B.relaxkv_shared_prefix_attention(*(a[k] for k in ("shape", "cache", "store", "rows", "q", "out", "workspace", "lse_out")), stream=0)


def sparse(a):
    B.relaxkv_block_sparse_attention(a["shape"], a["cache"], a["store"], a["rows"], 16, a["blocks"], a["q"], a["out"], a["workspace"], a["lse_out"], stream=0)


def select(a):
    B.relaxkv_select_blocks(a["shape"], 16, a["bounds"], a["scale"], a["rows"], a["q"], 1, 1, a["blocks"], a["workspace"], stream=0)


def bounds(a):
    B.relaxkv_block_bounds(a["shape"], a["cache"], 16, a["bounds"], a["scale"], stream=0)


FITS = {
    "rows of q": (dict(q=bf(6, 8, 64)), (shared, sparse, select)), "heads of q": (dict(q=bf(7, 4, 64)), (shared, sparse, select)),
    "type of q": (dict(q=bf(7, 8, 64).float()), (shared, sparse, select)), "order of q": (dict(q=bf(7, 12, 64)[:, :8]), (shared, sparse, select)),
    "rows of out": (dict(out=bf(6, 8, 64)), (shared, sparse)), "order of out": (dict(out=bf(8, 7, 64).transpose(0, 1)), (shared, sparse)),
    "rows of lse": (dict(lse_out=torch.zeros(8, 6)), (shared, sparse)), "order of lse": (dict(lse_out=torch.zeros(7, 8).t()), (shared, sparse)),
    "type of lse": (dict(lse_out=torch.zeros(8, 7, dtype=torch.float64)), (shared, sparse)),
    "rows of blocks": (dict(blocks=i32(6, 2, 4)), (sparse, select)), "heads of blocks": (dict(blocks=i32(7, 1, 4)), (sparse, select)),
    "type of blocks": (dict(blocks=torch.zeros(7, 2, 4, dtype=torch.int64)), (sparse, select)), "order of blocks": (dict(blocks=i32(7, 2, 6)[..., :4]), (sparse, select)),
    "bounds": (dict(bounds=torch.zeros(9, 2, 2, 64, dtype=torch.int8)), (select, bounds)), "scales": (dict(scale=torch.zeros(9, 2)), (select, bounds)),
    "type of bounds": (dict(bounds=torch.zeros(10, 2, 2, 64)), (select, bounds)),
    "contexts of rows": (dict(rows=step(ctx=(100, 33), seqs=(2, 3))["rows"]), (shared, sparse, select)),
    "heads of the cache": (dict(cache=step(Hkv=1)["cache"]), (shared, sparse, bounds)), "dim of the cache": (dict(cache=step(D=128)["cache"]), (shared, sparse, bounds)),
    "tokens of the cache": (dict(cache=step(ctx=(100, 0, 32))["cache"]), (shared, sparse, bounds)),
    "requests of the cache": (dict(cache=step(ctx=(100, 33), seqs=(2, 3))["cache"]), (shared, sparse, bounds)),
    "heads of the store": (dict(store=step(Hkv=1)["store"]), (shared, sparse)), "dim of the store": (dict(store=step(D=128)["store"]), (shared, sparse)),
}


@pytest.mark.parametrize("name", list(FITS))
def test_attention_refuses_what_does_not_fit_the_step(calls, name):
    kw, entries = FITS[name]
    for entry in entries:
        with pytest.raises(ValueError):
            entry(dict(step(), **kw))
    assert not calls


def test_attention_takes_what_it_took(calls):
    more = step(n_rows=9, Hkv=4)
    for kw in (dict(), dict(lse_out=None), dict(store=None), {k: more[k] for k in ("q", "out", "cache", "store")}, dict(bounds=torch.zeros(30, 2, 2, 64, dtype=torch.int8))):
        a = dict(step(), **kw)
        for entry, n in ((shared, 10), (sparse, 13), (select, 13), (bounds, 6)):
            entry(a)
            assert len(calls[-1][1]) == n
        assert calls[-4][1][4:7] == tuple(None if a[k] is None else a[k].data_ptr() for k in ("q", "out", "lse_out"))
        assert calls[-2][1][2:4] == (a["bounds"].data_ptr(), a["scale"].data_ptr()) and calls[-2][1][5:10] == (a["q"].data_ptr(), 4, 1, 1, a["blocks"].data_ptr())
        assert calls[-3][1][4:8] == (16, a["blocks"].data_ptr(), 4, a["q"].data_ptr()) and calls[-1][1][3:5] == (a["bounds"].data_ptr(), a["scale"].data_ptr())
    none = dict(step(ctx=(0, 0, 0)), cache=None)
    shared(none)
    sparse(none)
    assert [c[1][1] for c in calls[-2:]] == [None, None]
