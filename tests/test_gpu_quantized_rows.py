"""Many rows of a sequence over the 8-bit store (more (row, head) columns than one block of the kernel of few rows holds) against the plain 64-bit form."""
import numpy as np
import pytest
import torch

from tests import quantized_oracle as orc
from tests.test_gpu_quantized import B, attend, check, f64, i32, make_store, rnd, status, store_values, value_scale, workspace

pytestmark = pytest.mark.gpu


def check_rows(r, store, D, n):
    """The tolerance of few rows, but for what fp16's lowest step takes: the row's largest weight is at 2^11 or above, before it meets its value's scale, and scales are relative to
    the sequence's largest.  A weight times a scale is off by up to 2^-25, 2^-36 of the largest weight (1 at most, of a sum of weights of 1) times the largest scale, for each of n
    tokens and values of up to 448."""
    top = float(np.nanmax(value_scale(store)))
    r["wants"] = [(*w[:4], np.full_like(w[4], 2.0 ** -36 * n * 448 * top)) for w in r["wants"]]
    check(r, D)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,new,H,Hkv,D,block,layout", [
    ([1500], [40], 32, 8, 128, 16, "token"),            # more rows than a tile of them
    ([700, 33, 1300], [60, 33, 20], 4, 1, 64, 64, "head"),
    ([900], [300], 4, 4, 128, 32, "token"),             # one head a group: 128 rows a tile
    ([1400, 5], [50, 1], 16, 1, 128, 128, "head"),      # 16 heads a group: 8 rows a tile
    ([260, 129, 128, 127], [45, 40, 1, 127], 6, 2, 64, 16, "token"),      # three heads a group: two lanes of 128 are nobody's
    ([2100, 1], [64, 1], 10, 2, 128, 16, "head"),
    ([36] * 40, [36] * 40, 4, 2, 64, 16, "token"),      # a block has several tasks
])
def test_many_rows(lens, new, H, Hkv, D, block, layout, kind):
    n_blocks = sum(-(-t // block) for t in lens) + 3
    store = make_store(n_blocks, block, Hkv, D, kind, layout, seed=sum(lens))
    r = attend(store, lens, new, H, block, seed=len(lens), gaps=len(lens) > 1)
    check_rows(r, store, D, max(lens))
    assert status() == B().OK


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,new,H,Hkv,D", [
    ([300, 250], [3, 3], 16, 2, 128), ([2500, 1100], [4, 4], 20, 4, 128), ([1500, 40], [6, 5], 8, 2, 64), ([130], [24], 2, 2, 64), ([1300, 1200], [8, 7], 8, 2, 128), ([64, 31], [6, 6], 10, 2, 64),
    ([1030], [2], 16, 1, 128)])
def test_rows_of_three_and_four_column_tiles(lens, new, H, Hkv, D, kind):
    """17 to 32 columns: short sequences a block to each row tile and head, long ones in shares; what the largest calls of few rows take."""
    store = make_store(sum(-(-t // 16) for t in lens) + 2, 16, Hkv, D, kind, "head" if D == 64 else "token", seed=sum(lens))
    r = attend(store, lens, new, H, 16, seed=3, gaps=len(lens) > 1)
    check(r, D)
    assert status() == B().OK


def test_rows_that_see_nothing_and_sequences_without_tokens():
    """Rows before a sequence's first tokens (zeros and -inf), a sequence of rows without any token, one without rows."""
    store = make_store(20, 16, 2, 64, "int8", seed=4)
    lens, new, H = [100, 0, 50, 64], [110, 60, 0, 64], 8
    r = attend(store, lens, new, H, 16, seed=5)
    check_rows(r, store, 64, 100)
    out, lse = f64(r["out"]), f64(r["lse"])
    for rows in (slice(0, 10), slice(110, 170)):
        assert (out[rows] == 0).all() and (lse[:, rows] == -np.inf).all()
    assert status() == B().OK


def test_blocks_that_are_none_are_passed_over_by_many_rows():
    """A block number out of range: reported, its tokens weigh nothing, whatever shares their tile."""
    block, Hkv, H, D, T, n = 16, 2, 8, 128, 700, 40
    store = make_store(50, block, Hkv, D, "int8", seed=6)
    table = np.random.default_rng(1).permutation(50)[:44]
    table[[3, 4, 5, 6, 7, 8, 9, 10, 20, 43]] = [-1, 50, 2 ** 31 - 1, -2 ** 31, 51, -7, 50, 50, 99, -1]        # a whole tile of them among these
    q, out, lse = rnd(n, H, D, seed=7), torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(H, n, device="cuda")
    lens = [T - n + 1 + j for j in range(n)]
    rows = B().ContinuationRows([0, 1], [n], T, i32([0, n]), i32([0] * n), i32(lens), i32(table[None]))
    B().relaxkv_quantized_attention(store, rows, q, out, workspace(H, Hkv, D), lse_out=lse)
    assert status() == B().ERR_BAD_INDEX
    kk, vv = store_values(store)
    there = np.array([t for t in range(T) if 0 <= table[t // block] < 50])
    slots = table[there // block] * block + there % block
    seen = [int((there < x).sum()) for x in lens]
    want, want_lse, mass, most, lost = orc.attention(f64(q), kk[slots], vv[slots], seen, D ** -0.5, value_scale(store)[slots])
    tol, lse_tol = orc.attention_tolerance(want, want_lse, mass, most, lost + 2.0 ** -36 * T * 448 * value_scale(store).max(), D)
    assert (np.abs(f64(out) - want) <= tol).all() and (np.abs(f64(lse) - want_lse) <= lse_tol).all()


def test_what_is_no_number_stays_with_the_rows_that_see_it():
    """A NaN key or value reaches the rows that see it, of its head alone; a NaN row of Q is its own."""
    block, Hkv, H, D, T, n = 16, 2, 8, 64, 500, 48
    store = make_store(40, block, Hkv, D, "int8", seed=8)
    table = np.arange(32)
    for e, token, head in ((store.k_exp, T - 20, 0), (store.v_exp, T - 10, 1), (store.v_exp, T + 3, 0)):      # (the last: behind the sequence)
        e[int(table[token // block]), head, token % block] = -128
    q = rnd(n, H, D, seed=9)
    q[5, 6, 3], q[7, 1, 0] = float("nan"), float("inf")
    out, lse = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(H, n, device="cuda")
    lens = np.array([T - n + 1 + j for j in range(n)])
    rows = B().ContinuationRows([0, 1], [n], T, i32([0, n]), i32([0] * n), i32(lens), i32(table[None]))
    B().relaxkv_quantized_attention(store, rows, q, out, workspace(H, Hkv, D), lse_out=lse)
    bad = np.zeros((n, H), dtype=bool)
    bad[lens > T - 20, :4] = True
    bad[lens > T - 10, 4:] = True
    bad[5, 6] = bad[7, 1] = True
    got = torch.isnan(out).all(-1).cpu().numpy()
    assert (got == bad).all() and (np.isfinite(f64(out)).all(-1) == ~bad).all()
    assert status() == B().OK


def test_exponents_of_many_rows_from_end_to_end():
    """Values of every size side by side: those far below the largest of the sequence weigh what fp16 leaves of them, nothing overflows, and O is rescaled as they grow."""
    block, Hkv, H, D, T, n = 16, 1, 4, 64, 640, 40
    store = make_store(40, block, Hkv, D, "int8", seed=10)
    rng = np.random.default_rng(3)
    store.k_exp.copy_(i32(rng.integers(-12, -5, store.k_exp.shape)).to(torch.int8))
    store.v_exp.copy_(torch.arange(T, device="cuda").reshape(40, 1, 16).mul(200).div(T, rounding_mode="floor").sub(100).to(torch.int8))      # -100 to 99, rising
    r = attend(store, [T], [n], H, block, seed=11, width=40)
    check_rows(r, store, D, T)
    flipped = make_store(40, block, Hkv, D, "int8", seed=10)
    flipped.k_exp.copy_(store.k_exp)
    flipped.v_exp.copy_(store.v_exp.flip(0).flip(2))
    check_rows(attend(flipped, [T], [n], H, block, seed=11, width=40), flipped, D, T)
    assert status() == B().OK


@pytest.mark.parametrize("scale", [1e-6, 1.0, 40.0, 3e4])
def test_large_and_small_logits_of_many_rows(scale):
    """Logits of a size at which fp32 keeps few of their places: the row's sum and its weights lose the same."""
    store = make_store(60, 16, 2, 128, "int8", seed=12)
    r = attend(store, [900], [36], 8, 16, seed=13, scale=scale)
    check_rows(r, store, 128, 900)
    assert status() == B().OK


def test_many_rows_give_the_same_bits_every_time():
    """Forty calls in a row, with and without others between them, on two streams: no sum depends on who comes first."""
    store = make_store(400, 16, 4, 128, "e4m3", seed=14)
    lens, new = [3000, 700, 1900, 64], [70, 20, 300, 64]
    r = attend(store, lens, new, 16, 16, seed=15)
    check_rows(r, store, 128, 3000)
    want, want_lse = r["out"].clone(), r["lse"].clone()
    side = torch.cuda.Stream()
    for i in range(40):
        r["out"].zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side if i & 1 else torch.cuda.current_stream()):
            r["run"]()
        torch.cuda.current_stream().wait_stream(side)
        left = r["n"]
        assert torch.equal(r["out"][:left], want[:left]) and torch.equal(r["lse"][:, :left], want_lse[:, :left])
    assert status() == B().OK


def test_many_rows_in_a_graph():
    """Captured once, replayed over other tables and lengths of the same sizes."""
    store = make_store(120, 16, 2, 64, "int8", seed=16)
    r = attend(store, [800, 300], [40, 40], 8, 16, seed=17)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        r["run"]()
    r["out"].fill_(7.0)
    r["lse"].fill_(7.0)
    g.replay()
    check_rows(r, store, 64, 800)
    shorter = attend(store, [300, 800], [40, 40], 8, 16, seed=17, q=r["q"], width=r["rows"]._keep[5].shape[1], ws=r["ws"], max_len=800)
    for mine, other in zip(r["rows"]._keep[2:], shorter["rows"]._keep[2:]):
        mine.copy_(other)
    r["out"].fill_(7.0)
    r["lse"].fill_(7.0)
    g.replay()
    r["wants"] = shorter["wants"]
    check_rows(r, store, 64, 800)
    assert status() == B().OK


def test_rows_of_blocks_far_into_a_store():
    """Offsets that 32 bits do not hold: 2.3 GB of keys, blocks of both ends."""
    block, Hkv, H, D = 128, 8, 8, 128
    n_blocks = 2 ** 31 // (block * Hkv * D) + 1100
    values = [torch.zeros(n_blocks, block, Hkv, D, dtype=torch.int8, device="cuda") for _ in range(2)]
    exps = [torch.full((n_blocks, Hkv, block), -7, dtype=torch.int8, device="cuda") for _ in range(2)]
    small = make_store(6, block, Hkv, D, "int8", seed=18)
    at = torch.tensor([0, n_blocks - 1, n_blocks - 2, 1, n_blocks // 2, n_blocks - 1000], device="cuda")
    for big, few in zip([*values, *exps], (small.k, small.v, small.k_exp, small.v_exp)):
        big[at] = few
    store = B().QuantizedStore(*values, *exps)
    T = 6 * block - 5
    for n in (1, 3, 50):
        q, outs, lses = rnd(n, H, D, seed=n), [], []
        for s, ids in ((store, at.tolist()), (small, list(range(6)))):
            outs.append(torch.empty_like(q))
            lses.append(torch.empty(H, n, device="cuda"))
            rows = B().ContinuationRows([0, 1], [n], T, i32([0, n]), i32([0] * n), i32([T - n + 1 + j for j in range(n)]), i32([ids]))
            B().relaxkv_quantized_attention(s, rows, q, outs[-1], workspace(H, Hkv, D), lse_out=lses[-1])
        assert torch.equal(*outs) and torch.equal(*lses)
    slots = (at[:, None] * block + torch.arange(block, device="cuda")).reshape(-1)[:T].to(torch.int32)
    k, v = (torch.empty(T, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B().relaxkv_read_quantized(store, slots, k, v)
    kk, vv = store_values(small)
    assert (f64(k) == kk[:T]).all() and (f64(v) == vv[:T]).all()
    B().relaxkv_append_quantized(store, v, k, slots)
    back = [torch.empty_like(k), torch.empty_like(v)]
    B().relaxkv_read_quantized(store, slots, *back)
    assert torch.equal(back[0], v) and torch.equal(back[1], k) and status() == B().OK


def test_calls_at_once_on_two_streams():
    """Many rows on one stream, few rows, an append and a matrix product on another, each with its own workspace: every call gives what it gives by itself."""
    store, other = make_store(300, 16, 4, 128, "int8", seed=20), make_store(300, 16, 4, 128, "e4m3", seed=21)
    many = attend(store, [2000, 900], [70, 90], 16, 16, seed=22)
    few = attend(other, [1500, 300, 40], [3, 2, 1], 16, 16, seed=23)
    check_rows(many, store, 128, 2000)
    check(few, 128)
    w, x, y = rnd(1024, 512, seed=24, scale=0.05), rnd(300, 512, seed=25), torch.empty(300, 1024, dtype=torch.bfloat16, device="cuda")
    B().relaxkv_linear(x, w, y)
    spare = B().QuantizedStore.empty(4, 16, 4, 128, device="cuda")
    k, v = rnd(50, 4, 128, seed=26), rnd(50, 4, 128, seed=27)
    B().relaxkv_append_quantized(spare, k, v, i32(range(50)))
    torch.cuda.synchronize()
    want = [t.clone() for t in (many["out"], many["lse"], few["out"], few["lse"], y, spare.k, spare.k_exp)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(50):
        many["run"]()
        with torch.cuda.stream(side):
            few["run"]()
            B().relaxkv_linear(x, w, y)
            B().relaxkv_append_quantized(spare, k, v, i32(range(50)))
    torch.cuda.synchronize()
    for a, b in zip((many["out"], many["lse"], few["out"], few["lse"], y, spare.k, spare.k_exp), want):
        assert torch.equal(a, b)
    assert status() == B().OK
