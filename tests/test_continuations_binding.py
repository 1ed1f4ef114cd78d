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
