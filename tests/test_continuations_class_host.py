"""What the class Continuations refuses before a call (buffers on the host; the calls that would be made are recorded, none runs)."""
import pytest
import torch

from paper_2609_33503_b200 import binding as B
from paper_2609_33503_b200 import inputs
from paper_2609_33503_b200.continuations import Continuations
from tests.test_continuations_binding import Recorder, bf

H, HKV, D, L = 8, 2, 64, 2
BLK = inputs.BlockShape(hidden=256, inter=384, rope_theta=1.0e4, eps=1.0e-5)


def make(monkeypatch, **kw):
    c = Continuations(H, HKV, D, (70,), (3,), L, BLK, n_blocks=20, max_len=40, block_size=16, max_rows=12, device="cpu", **kw)
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    return c, r.calls


def weights():
    C = BLK.hidden
    return [dict(w_in_norm=bf(C), w_post_norm=bf(C), w_qkv=bf((H + 2 * HKV) * D, C), wo=bf(C, H * D), w_gate_up=bf(2 * BLK.inter, C), w_down=bf(C, BLK.inter))
            for _ in range(L)]


def caches():
    return [B.CacheView(bf(70, HKV, D), bf(70, HKV, D), [0]) for _ in range(L)]


@pytest.mark.parametrize("h", [bf(4, 256), bf(5, 255), bf(5, 256).float(), bf(256, 5).t(), bf(5, 512)[:, :256], bf(5 * 256)], ids=["rows", "hidden", "type", "order", "slice", "dims"])
def test_a_step_refuses_other_rows_than_it_has(monkeypatch, h):
    c, calls = make(monkeypatch)
    assert c.begin([3, 1, 1]) == 5
    n = len(calls)
    with pytest.raises(ValueError):
        c.run(h, weights(), caches())
    assert len(calls) == n


def test_rows_behind_a_steps_own_are_not_looked_at(monkeypatch):
    c, calls = make(monkeypatch, n_select=2)
    c.begin([3, 1, 1])
    calls.clear()
    assert c.run(bf(40, 256), weights(), caches()).shape == (5, 256)
    names = [name for name, _ in calls]
    assert names.count("relaxkv_rmsnorm") == 2 * L and all(a[3] == 5 for name, a in calls if name == "relaxkv_rmsnorm")
    lists = [a[9] if name == "relaxkv_select_blocks" else a[5] for name, a in calls if name in ("relaxkv_select_blocks", "relaxkv_block_sparse_attention")]
    assert lists == [c.blocks.data_ptr()] * 2 * L


def test_attention_refuses_other_rows_than_the_step_has(monkeypatch):
    c, calls = make(monkeypatch, n_select=2)
    c.begin([3, 1, 1])
    calls.clear()
    with pytest.raises(ValueError):
        c.attention(0, caches()[0], bf(4, H, D), bf(5, H, D))
    with pytest.raises(ValueError):
        c.attention(0, caches()[0], bf(5, H, D), bf(4, H, D))
    assert [name for name, _ in calls] in (["relaxkv_select_blocks"], [])


@pytest.mark.parametrize("h,head,logits", [((13, 256), (104, 256), (13, 104)), ((5, 256), (104, 255), (5, 104)), ((5, 256), (104, 256), (4, 104)), ((5, 128), (104, 256), (5, 104))])
def test_the_output_head_refuses_more_rows_than_its_buffers_hold(monkeypatch, h, head, logits):
    c, calls = make(monkeypatch)
    with pytest.raises(ValueError):
        c.output_head(bf(*h), bf(256), bf(*head), bf(*logits))
    with pytest.raises(ValueError):
        c.output_head(bf(5, 256), bf(256), bf(104, 256), torch.zeros(5, 104))
    assert not calls
    c.output_head(bf(12, 256), bf(256), bf(104, 256), bf(20, 104))
    assert len(calls) == 2


def test_sequences_without_contexts_have_no_bounds_to_make(monkeypatch):
    """No context, no cache: as the attention calls take it."""
    c = Continuations(H, HKV, D, (0, 0), (1, 2), L, BLK, n_blocks=20, max_len=40, block_size=16, device="cpu", n_select=4)
    r = Recorder()
    monkeypatch.setattr(B, "lib", lambda: r)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    c.context_bounds([None] * L)
    assert [(name, a[1]) for name, a in r.calls] == [("relaxkv_block_bounds", None)] * L
    c.begin([1, 1, 1])
    assert c.run(bf(3, 256), weights(), [None] * L).shape == (3, 256)
