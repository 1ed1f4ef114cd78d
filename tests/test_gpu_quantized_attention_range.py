"""Attention over the 8-bit store at the ends of its documented range: exponents, queries that are no numbers, tokens that a row does not see."""
import numpy as np
import pytest
import torch

from tests import quantized_oracle as orc
from tests.test_gpu_quantized import B, attend, check, f64, i32, make_store, rnd, status, store_values, value_scale, workspace
from tests.test_gpu_quantized_rows import check_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,new", [([3, 0], [5, 2]), ([2000, 0], [2, 1]), ([100, 0, 700], [110, 60, 30]), ([4000, 0], [40, 40])])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_no_number_weighs_nothing_where_nothing_is_seen(lens, new, bad):
    """Zeros and -inf for a row without tokens, whatever its query; NaN for one that sees a token; the others as they were."""
    Hkv, D, block, H = 2, 64, 16, 8
    store = make_store(sum(-(-t // block) for t in lens) + 2, block, Hkv, D, "int8", seed=1)
    r = attend(store, lens, new, H, block, seed=3)
    clean = r["out"].clone(), r["lse"].clone()
    row_len = r["rows"]._keep[4]
    hit = torch.zeros(r["n"], dtype=torch.bool, device="cuda")
    hit[::2] = True
    empty = row_len[:r["n"]] == 0
    assert (hit & empty).any() and (hit & ~empty).any()
    r["q"][:r["n"]][hit] = bad
    r["out"].fill_(7)
    r["lse"].fill_(7)
    r["run"]()
    out, lse = r["out"][:r["n"]], r["lse"][:, :r["n"]]
    assert (out[empty] == 0).all() and (lse[:, empty] == -float("inf")).all()
    assert torch.isnan(out[hit & ~empty]).all() and torch.isnan(lse[:, hit & ~empty]).all()
    assert torch.equal(out[~hit], clean[0][:r["n"]][~hit]) and torch.equal(lse[:, ~hit], clean[1][:, :r["n"]][:, ~hit]) and status() == B().OK


@pytest.mark.parametrize("T,n", [(90, 2), (90, 40), (300, 60)])
def test_a_query_that_is_no_number_over_blocks_that_are_none(T, n):
    """All of a sequence's blocks out of range: reported, and its rows see nothing."""
    Hkv, D, block, H = 2, 64, 16, 8
    store = make_store(20, block, Hkv, D, "int8", seed=1)
    q = torch.full((n, H, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 7), torch.full((H, n), 7.0, device="cuda")
    rows = B().ContinuationRows([0, 1], [n], T, i32([0, n]), i32([0] * n), i32([T - n + 1 + j for j in range(n)]), i32([[-1] * 19]))
    B().relaxkv_quantized_attention(store, rows, q, out, workspace(H, Hkv, D), lse_out=lse)
    assert status() == B().ERR_BAD_INDEX and (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,new", [([250, 3], [2, 1]), ([3000, 40], [2, 2]), ([700, 90], [6, 5]), ([700], [40]), ([3000, 200], [60, 33])])
def test_keys_of_the_largest_exponents(lens, new, kind):
    """Keys up to 127 * 2^127 and queries as small: logits of ordinary size, in both kernels; others that only just weigh beside them."""
    Hkv, D, block, H = 1, 64, 16, 4
    store = make_store(sum(-(-t // block) for t in lens) + 1, block, Hkv, D, kind, seed=1)
    rng = np.random.default_rng(0)
    for low in (127, 121, 96):
        store.k_exp.copy_(i32(rng.integers(low, 128, tuple(store.k_exp.shape))).to(torch.int8))
        r = attend(store, lens, new, H, block, q=rnd(sum(new) + 2, H, D, seed=4, scale=2.0 ** -120), scale=2.0 ** -12 if kind == "int8" else 2.0 ** -14)
        check_rows(r, store, D, max(lens))
    store.k_exp.fill_(127)
    store.k.view(torch.int8).zero_()                                        # elements of nothing, whatever their exponent
    check_rows(attend(store, lens, new, H, block), store, D, max(lens))
    assert status() == B().OK


@pytest.mark.parametrize("lens,new", [([250, 3], [2, 1]), ([700, 20], [40, 30])])
@pytest.mark.parametrize("q_scale,scale", [(0.0, 0.125), (0.0, 1e-12), (2.0 ** -110, 1e-12), (2.0 ** -110, 1e-30), (1.0, 1e-30)])
def test_logits_of_nothing(lens, new, q_scale, scale):
    """Queries or scales so small that all logits are nothing: what is seen weighs alike, what is not seen nothing."""
    Hkv, D, block, H = 2, 64, 16, 8
    store = make_store(sum(-(-t // block) for t in lens) + 1, block, Hkv, D, "int8", seed=2)
    r = attend(store, lens, new, H, block, q=rnd(sum(new) + 2, H, D, seed=4, scale=q_scale), scale=scale)
    check_rows(r, store, D, max(lens))
    assert status() == B().OK


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("T,n,H,Hkv,D", [(650, 40, 8, 2, 128), (640, 40, 8, 2, 64), (5000, 60, 4, 1, 128), (130, 130, 4, 2, 64), (1290, 200, 2, 1, 128)])
def test_tokens_behind_a_row_take_none_of_its_bits(T, n, H, Hkv, D, kind):
    """Values behind a row, up to 2^190 times as large as those that it sees: its weights are rounded relative to what it sees."""
    block = 16
    store = make_store(-(-T // block) + 2, block, Hkv, D, kind, seed=T)
    ids = np.random.default_rng(3).permutation(store.k.shape[0])[:-(-T // block)]              # (the blocks that attend() hands out)
    low = -90 if D == 64 else -9
    store.v_exp.add_(low + 9)
    for token, e in ((T - 37, 5), (T - 25, 30), (T - 12, 70), (T - 10, 60), (T - 2, 100)):
        store.v_exp[int(ids[token // block]), :, token % block] = e
    r = attend(store, [T], [n], H, block, seed=3)
    slots = (r["keep"][0][0, :len(ids), None] * block + np.arange(block)).reshape(-1)[:T].astype(int)
    top = np.maximum.accumulate(value_scale(store)[slots], 0)               # [T, H_kv]: of what a row of so many tokens sees
    lens = [max(0, T - n + 1 + j) for j in range(n)]
    want, lse, mass, most, _ = r["wants"][0]
    # the row's largest weight is at 2^11 or above before it meets its value's scale: off by up to 2^-36 of the largest weight times the largest scale that the row sees, for each of its
    # tokens and values of up to 448
    lost = 2.0 ** -36 * T * 448 * np.stack([top[max(t, 1) - 1].repeat(H // Hkv) * (t > 0) for t in lens], 1)
    r["wants"] = [(want, lse, mass, most, lost)]
    check(r, D)
    assert status() == B().OK


@pytest.mark.parametrize("lens,new", [([250, 3], [2, 1]), ([3000, 40], [2, 2]), ([700, 90], [6, 5]), ([700, 90], [40, 30])])
def test_queries_of_the_largest_numbers(lens, new):
    """Queries up to bf16's largest number over keys as small: logits of ordinary size, and queries of ordinary size beside them."""
    Hkv, D, block, H = 1, 64, 16, 4
    store = make_store(sum(-(-t // block) for t in lens) + 1, block, Hkv, D, "int8", seed=1)
    store.k_exp.fill_(-100)
    for power, scale in ((124, 2.0 ** -34), (112, 2.0 ** -22)):
        q = rnd(sum(new) + 2, H, D, seed=4, scale=2.0 ** power)
        q[:, 1] = rnd(sum(new) + 2, D, seed=5)
        assert torch.isfinite(q).all()
        check_rows(attend(store, lens, new, H, block, q=q, scale=scale), store, D, max(lens))
    q[0, 2, 3] = torch.finfo(torch.bfloat16).max
    check_rows(attend(store, lens, new, H, block, q=q, scale=2.0 ** -40), store, D, max(lens))
    # logits of 2^31 and more: one key's weight alone, whichever fp32 finds the largest; a score is off by its sums' roundings, (D + 8) 2^-24 of the sum of its products' sizes
    q[:, 1] = 0
    r = attend(store, lens, new, H, block, q=q)
    out, lse = f64(r["out"]), f64(r["lse"])
    assert np.isfinite(out).all()
    for (_, want, _, most, _), a, b in zip(r["wants"], r["cu"], r["cu"][1:]):
        assert (np.abs(lse[:, a:b] - want) <= (D + 8) * 2.0 ** -24 * most + 2.0 ** -18 + 2.0 ** -21 * np.abs(want)).all()
    assert status() == B().OK


def test_a_value_that_is_no_number_beside_tokens_that_are_not_seen():
    """A row that sees tokens 2^130 times smaller than those behind it, the last of them NaN."""
    T, n, H, D, block = 128, 64, 4, 64, 16
    store = make_store(8, block, 1, D, "int8", seed=1)
    store.v_exp.copy_(i32([-90] * 64 + [-128] + [40] * 63).to(torch.int8).view(8, 1, block))
    q, out, lse = rnd(n, H, D, seed=2), torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(H, n, device="cuda")
    lens = [T - n + 1 + j for j in range(n)]
    rows = B().ContinuationRows([0, 1], [n], T, i32([0, n]), i32([0] * n), i32(lens), i32([list(range(8))]))
    for _ in range(3):
        B().relaxkv_quantized_attention(store, rows, q, out, workspace(H, 1, D), lse_out=lse)
        assert torch.isnan(out).all() and torch.isfinite(lse).all()
    store.v_exp[4, 0, 0] = -90
    kk, vv = store_values(store)
    B().relaxkv_quantized_attention(store, rows, q, out, workspace(H, 1, D), lse_out=lse)
    want, want_lse, mass, most, _ = orc.attention(f64(q), kk, vv, lens, D ** -0.5)
    top = np.maximum.accumulate(value_scale(store)[:, 0])[np.array(lens) - 1]
    tol, lse_tol = orc.attention_tolerance(want, want_lse, mass, most, 2.0 ** -36 * T * 448 * np.tile(top, (H, 1)), D)
    assert (np.abs(f64(out) - want) <= tol).all() and (np.abs(f64(lse) - want_lse) <= lse_tol).all() and status() == B().OK


@pytest.mark.parametrize("kind,e", [("int8", 120), ("e4m3", 118)])
@pytest.mark.parametrize("lens,new", [([250, 3], [2, 1]), ([3000, 40], [2, 2]), ([900], [50]), ([4000], [33])])
def test_values_of_the_largest_numbers(lens, new, kind, e):
    """Outputs of up to 2^127, joined from several parts: no sum on the way leaves fp32."""
    Hkv, D, block, H = 1, 64, 16, 4
    store = make_store(sum(-(-t // block) for t in lens) + 1, block, Hkv, D, kind, seed=1)
    store.v_exp.fill_(e)
    store.v.view(torch.int8).fill_(127 if kind == "int8" else 0x7d)         # 127, 416
    check_rows(attend(store, lens, new, H, block), store, D, max(lens))
    assert status() == B().OK
