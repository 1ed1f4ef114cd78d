"""Rotary embeddings of every form and contexts kept in 8 bits on the GPU against their plain 64-bit forms (tests/quantized_oracle.py)."""
import numpy as np
import pytest
import torch

from tests import quantized_oracle as orc

pytestmark = pytest.mark.gpu
TYPES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def B():
    from paper_2609_33503_b200 import binding
    return binding


def status():
    torch.cuda.synchronize()
    return B().relaxkv_read_device_status()[0]


def i32(xs):
    return torch.tensor(np.asarray(xs).tolist(), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().float().double().cpu().numpy()


def rnd(*shape, seed, scale=1.0):
    return (scale * torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")).to(torch.bfloat16)


def workspace(H, Hkv, D):
    nbytes = B().relaxkv_quantized_workspace_bytes(H, Hkv, D)
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda").fill_(255)                # NaN, whatever is read before it is written
    off = (-ws.data_ptr()) % 256
    return ws[off:off + nbytes]


def laid_out(x, layout):
    return x.transpose(-3, -2).contiguous().transpose(-3, -2) if layout == "head" else x.contiguous()


def make_store(n_blocks, block, Hkv, D, kind, layout="token", seed=0, junk=False):
    """A store of random values; junk: bytes and exponents of every kind, NaN among them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = [torch.randint(-128 if junk else -127, 128, (n_blocks, block, Hkv, D), generator=g, device="cuda").to(torch.int8) for _ in range(2)]
    if kind == "e4m3" and not junk:
        v = [torch.where((x & 127) == 127, 5, x).to(torch.int8) for x in v]
    e = [torch.randint(-128 if junk else -9, 128 if junk else -4, (n_blocks, Hkv, block), generator=g, device="cuda").to(torch.int8) for _ in range(2)]
    return B().QuantizedStore(*(laid_out(x, layout).view(TYPES[kind]) for x in v), *e)


def store_values(store):
    """K, V [n_blocks * block, H_kv, D] in 64 bits."""
    out = []
    for v, e in ((store.k, store.k_exp), (store.v, store.v_exp)):
        out.append(orc.values(f64(v), e.cpu().numpy().astype(np.int64).transpose(0, 2, 1)).reshape(-1, store.heads, store.dim))
    return out


def value_scale(store):
    """2^exponent of the values, [n_blocks * block, H_kv]."""
    return 2.0 ** store.v_exp.cpu().numpy().astype(np.float64).transpose(0, 2, 1).reshape(-1, store.heads)


def store_bytes(store):
    return [x.view(torch.int8).clone() for x in (store.k, store.v, store.k_exp, store.v_exp)]


def rotary(part, pairs, amplitude=1.0):
    r = B().Rotary.scaled(part, 1e5, "bands", 4.0, 4096, 1.0, 4.0, interleaved=pairs == "interleaved")
    return B().Rotary(r.freq, r.interleaved, amplitude)


def rotation_tolerance(x, want, w, amplitude):
    """fp32: sine and cosine are off by 2^-22 (argument to 2^-24 of a turn: 2^-21.3 radians), a norm by some 2^-20 of its values; the pair's larger element bounds both.  Then
    one rounding to bf16."""
    top = np.abs(want).max(-1, keepdims=True) if w is not None else np.abs(x).max(-1, keepdims=True) * 1.5 * amplitude
    return 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * top


# ---- rotation ----

@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("n,H,Hkv,D,part,norm,amplitude", [
    (1, 4, 1, 64, 64, False, 1.0), (3, 4, 1, 64, 8, True, 1.25), (65, 32, 8, 128, 128, False, 1.0), (7, 40, 8, 128, 64, True, 1.2), (1190, 24, 8, 128, 104, True, 1.0),
    (1203, 32, 8, 64, 40, False, 0.9), (2500, 4, 1, 64, 16, True, 1.0), (33, 1, 1, 128, 24, True, 1.1), (5, 17, 3, 128, 120, False, 1.0)])
def test_rotation(n, H, Hkv, D, part, norm, amplitude, pairs):
    q, k = rnd(n, H, D, seed=1), rnd(n, Hkv, D, seed=2)
    wq, wk = (1 + rnd(D, seed=3 + i, scale=0.2) if norm else None for i in range(2))
    pos = torch.randint(-70000, 70000, (n,), generator=torch.Generator().manual_seed(5)).to(torch.int32)
    rot, qo, ko = rotary(part, pairs, amplitude), torch.empty_like(q), torch.empty_like(k)
    B().relaxkv_qk_norm_rotate(q, k, pos.cuda(), rot, qo, ko, wq, wk, 1e-5)
    for x, got, w in ((q, qo, wq), (k, ko, wk)):
        want = orc.turned(f64(x), None if w is None else f64(w), 1e-5, pos.numpy(), rot.freq.cpu().numpy(), pairs == "interleaved", rot.amplitude)
        assert (np.abs(f64(got) - want) <= rotation_tolerance(f64(x), want, w, amplitude)).all()
        if not norm:
            assert torch.equal(got[..., part:], x[..., part:])
    qi, ki = q.clone(), k.clone()
    B().relaxkv_qk_norm_rotate(qi, ki, pos.cuda(), rot, w_q_norm=wq, w_k_norm=wk, eps=1e-5)                       # in place
    assert torch.equal(qi, qo) and torch.equal(ki, ko)
    one = torch.empty_like(k)
    B().relaxkv_qk_norm_rotate(None, k, pos.cuda(), rot, None, one, wq, wk, 1e-5)                                 # keys alone
    assert torch.equal(one, ko)
    two = torch.empty_like(q)
    B().relaxkv_qk_norm_rotate(q, None, pos.cuda(), rot, two, None, wq, wk, 1e-5)
    assert torch.equal(two, qo) and status() == B().OK


@pytest.mark.parametrize("pairs", ["half", "interleaved"])
def test_rotation_of_parts_of_larger_rows(pairs):
    """Queries and keys of fused rows, in place: nothing beside them changes; keys of a head-major cache."""
    n, H, Hkv, D = 37, 6, 2, 128
    fused = rnd(n, (H + 2 * Hkv) * D + 8, seed=1)
    before = fused.clone()
    heads = fused[:, 8:].unflatten(1, (-1, D))
    q, k = heads[:, :H], heads[:, H:H + Hkv]
    pos, rot = torch.arange(n, dtype=torch.int32, device="cuda"), rotary(96, pairs)
    want_q, want_k = torch.empty(n, H, D, dtype=q.dtype, device="cuda"), torch.empty(n, Hkv, D, dtype=q.dtype, device="cuda")
    B().relaxkv_qk_norm_rotate(q.contiguous(), k.contiguous(), pos, rot, want_q, want_k)
    B().relaxkv_qk_norm_rotate(q, k, pos, rot)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(fused[:, :8], before[:, :8])
    assert torch.equal(heads[:, H + Hkv:], before[:, 8:].unflatten(1, (-1, D))[:, H + Hkv:])
    cache = laid_out(k, "head")
    B().relaxkv_qk_norm_rotate(None, cache, -pos, rot)
    back = f64(before[:, 8:].unflatten(1, (-1, D))[:, H:H + Hkv])
    # there and back: two roundings to bf16 of values of the pair's size
    assert (np.abs(f64(cache) - back) <= 2.0 ** -7 * 1.5 * np.abs(back).max(-1, keepdims=True)).all() and status() == B().OK


def test_rotation_agrees_with_the_plain_call():
    """The half form of the whole head with unscaled frequencies is what relaxkv_qk_norm_rope does, whose normed values take one rounding more."""
    n, H, Hkv, D = 100, 8, 2, 128
    q, k, w = rnd(n, H, D, seed=1), rnd(n, Hkv, D, seed=2), 1 + rnd(D, seed=3, scale=0.1)
    pos = torch.arange(1000, 1000 + n, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(k)
    B().relaxkv_qk_norm_rotate(q, k, pos, B().Rotary.scaled(D, 1e6), a, b)
    B().relaxkv_qk_norm_rope(q, k, pos, 1e6)
    for x, y in ((a, q), (b, k)):
        assert (np.abs(f64(x) - f64(y)) <= 2.0 ** -7 * np.abs(f64(x)) + 2.0 ** -18 * 10).all()
    assert status() == B().OK


def test_far_positions():
    """Up to the last position that 32 bits hold; a frequency of one radian, the fastest there is: the product's rounding in 64 bits is 2^-22 of a turn."""
    q = rnd(4, 1, 64, seed=1)
    pos = np.array([2 ** 31 - 1, -2 ** 31, 1_000_003, 0])
    rot = B().Rotary(torch.linspace(1, 0.1, 32, dtype=torch.float64, device="cuda"))
    out = torch.empty_like(q)
    B().relaxkv_qk_norm_rotate(q, None, torch.tensor(pos, dtype=torch.int32, device="cuda"), rot, out)
    want = orc.turned(f64(q), None, 0, pos, rot.freq.cpu().numpy(), False, 1.0)
    assert (np.abs(f64(out) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -18 * np.abs(f64(q)).max() * 2).all()
    assert torch.equal(out[3], q[3])


def test_dims_that_stay_keep_what_is_no_number():
    q = rnd(2, 2, 64, seed=1)
    q[0, 0, 40], q[0, 1, 63], q[1, 0, 3] = float("inf"), float("nan"), float("inf")
    out = torch.empty_like(q)
    B().relaxkv_qk_norm_rotate(q, None, i32([5, 6]), rotary(32, "half"), out)
    assert torch.equal(out[..., 32:].view(torch.int16), q[..., 32:].view(torch.int16)) and torch.isfinite(out[0, :, :32]).all()
    bad = ~torch.isfinite(out[1, 0])
    assert bad.nonzero().flatten().tolist() == [3, 19] and torch.isfinite(out[1, 1]).all()


# ---- writing ----

def written(store, slots):
    """Values and exponents at slots, as numbers: ([n, H_kv, D], [n, H_kv]) of K and of V."""
    s = np.asarray(slots)
    return [(f64(v)[s // store.block_size, s % store.block_size], e.cpu().numpy().astype(np.int64).transpose(0, 2, 1)[s // store.block_size, s % store.block_size])
            for v, e in ((store.k, store.k_exp), (store.v, store.v_exp))]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,Hkv,D,block,layout", [(1, 1, 64, 16, "token"), (5, 8, 128, 16, "head"), (130, 2, 128, 32, "token"), (1500, 8, 64, 64, "head"), (2000, 3, 128, 128, "token")])
def test_rows_are_written_as_they_are(n, Hkv, D, block, layout, kind):
    n_blocks = n // block + 3
    st = make_store(n_blocks, block, Hkv, D, kind, layout)
    before = store_bytes(st)
    slots = np.random.default_rng(n).permutation(n_blocks * block)[:n]
    size = torch.exp2(torch.randint(-30, 30, (n, Hkv, 1), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").float())
    k, v = ((rnd(n, Hkv, D, seed=2 + i).float() * size).to(torch.bfloat16) for i in range(2))
    k[0, 0, 1:] = 0                                                        # a row of one element, of none, of ties
    v[0] = 0
    v[-1, -1] = torch.arange(D, device="cuda").to(torch.bfloat16) - 31.5
    k, v = laid_out(k, layout), laid_out(v, layout)
    B().relaxkv_append_quantized(st, k, v, i32(slots))
    for x, (got, e) in zip((k, v), written(st, slots)):
        want, want_e = orc.quantized(f64(x), kind)
        assert np.array_equal(e, want_e) and np.array_equal(got, want)
    rest = np.setdiff1d(np.arange(n_blocks * block), slots)
    for a, b in zip(before[:2], store_bytes(st)[:2]):
        assert torch.equal(a[rest // block, rest % block], b[rest // block, rest % block])
    for a, b in zip(before[2:], store_bytes(st)[2:]):
        assert torch.equal(a.transpose(1, 2)[rest // block, rest % block], b.transpose(1, 2)[rest // block, rest % block])
    assert status() == B().OK


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("pairs", ["half", "interleaved"])
@pytest.mark.parametrize("n,H,Hkv,D,part,norm", [(1, 4, 1, 64, 64, False), (64, 32, 8, 128, 128, True), (1301, 40, 8, 128, 48, True), (9, 5, 5, 64, 24, False)])
def test_rows_are_turned_and_written(n, H, Hkv, D, part, norm, pairs, kind):
    block = 16
    st = make_store(n // block + 2, block, Hkv, D, kind)
    q, k, v = rnd(n, H, D, seed=1), rnd(n, Hkv, D, seed=2), rnd(n, Hkv, D, seed=3)
    wq, wk = (1 + rnd(D, seed=4 + i, scale=0.2) if norm else None for i in range(2))
    pos = torch.randint(0, 60000, (n,), generator=torch.Generator().manual_seed(6)).to(torch.int32)
    rot, slots, qo = rotary(part, pairs, 1.125), np.arange(n)[::-1] + 3, torch.empty_like(q)
    B().relaxkv_append_quantized(st, k, v, i32(slots), q=q, q_out=qo, positions=pos.cuda(), rotary=rot, w_q_norm=wq, w_k_norm=wk, eps=1e-6)
    args = (1e-6, pos.numpy(), rot.freq.cpu().numpy(), pairs == "interleaved", 1.125)
    want_q = orc.turned(f64(q), None if wq is None else f64(wq), *args)
    assert (np.abs(f64(qo) - want_q) <= rotation_tolerance(f64(q), want_q, wq, 1.125)).all()
    want_k = orc.turned(f64(k), None if wk is None else f64(wk), *args)
    (kv, ke), (vv, ve) = written(st, slots)
    want_v, want_ve = orc.quantized(f64(v), kind)
    assert np.array_equal(vv, want_v) and np.array_equal(ve, want_ve)
    # keys: the exponent is the definition's for the largest value give or take fp32's error of it; values are within half a step of the turned key and that error
    slop = 2.0 ** -18 * 1.5 * 1.125 * np.abs(want_k).max(-1)
    lo, hi = (np.array([[orc.exponent(max(t, 0.0), orc.MOST[kind]) for t in r] for r in np.abs(want_k).max(-1) + d]) for d in (-slop, slop))
    assert ((ke >= lo) & (ke <= hi)).all()
    scale = 2.0 ** ke[..., None].astype(np.float64)
    step = scale if kind == "int8" else scale * np.exp2(np.floor(np.log2(np.maximum(np.abs(want_k) / scale * (1 + 2.0 ** -16), 2.0 ** -6))) - 3)
    assert (np.abs(kv * scale - want_k) <= step / 2 + slop[..., None]).all()
    # the call without queries, and without keys' rotation, writes what this one has
    other = make_store(n // block + 2, block, Hkv, D, kind)
    B().relaxkv_append_quantized(other, k, v, i32(slots), positions=pos.cuda(), rotary=rot, w_q_norm=wq, w_k_norm=wk, eps=1e-6)
    assert all(torch.equal(a, b) for a, b in zip(store_bytes(st), store_bytes(other))) and status() == B().OK


@pytest.mark.parametrize("kind", list(TYPES))
def test_what_is_no_number_and_the_ends_of_the_range(kind):
    k = torch.zeros(8, 1, 64, dtype=torch.bfloat16, device="cuda")
    k[0, 0, 3], k[1, 0, 63], k[2, 0, 0] = float("nan"), float("inf"), -float("inf")
    k[3, 0, 7], k[4, 0, 5] = torch.finfo(torch.bfloat16).max, -torch.finfo(torch.bfloat16).max
    k[5, 0, 2], k[6, 0, 2] = 2.0 ** -133, 2.0 ** -94
    k[:3, 0, 10] = 1.0
    st = make_store(1, 16, 1, 64, kind)
    B().relaxkv_append_quantized(st, k, k, i32(range(8)))
    for got, e in written(st, range(8)):
        want, want_e = orc.quantized(f64(k), kind)
        assert np.array_equal(e, want_e) and np.array_equal(got, want) and e[:3, 0].tolist() == [-128] * 3 and e[5:, 0].tolist() == [-100] * 3
    out = [torch.empty_like(k) for _ in range(2)]
    B().relaxkv_read_quantized(st, i32(range(8)), *out)
    assert torch.isnan(out[0][:3]).all() and torch.equal(out[0][3:].isnan(), torch.zeros(5, 1, 64, dtype=torch.bool, device="cuda")) and status() == B().OK


@pytest.mark.parametrize("pairs", [None, "half"])
def test_rows_without_a_slot_and_slots_outside(pairs):
    n, block = 6, 16
    st = make_store(2, block, 2, 64, "int8")
    before = store_bytes(st)
    q, k = rnd(n, 4, 64, seed=1), rnd(n, 2, 64, seed=2)
    qo = torch.zeros_like(q)
    kw = dict(positions=i32(range(n)), rotary=rotary(64, pairs)) if pairs else {}
    B().relaxkv_append_quantized(st, k, k, i32([-1, 5, -1, -1, -1, -1]), q=q, q_out=qo, **kw)
    assert status() == B().OK and (qo != 0).any(-1).all()                   # rows without a slot are turned
    for bad in (32, -2, 2 ** 31 - 1):
        now = store_bytes(st)
        B().relaxkv_append_quantized(st, k, k, i32([-1, -1, bad, -1, -1, -1]), q=q, q_out=qo, **kw)
        assert status() == B().ERR_BAD_INDEX and all(torch.equal(a, b) for a, b in zip(now, store_bytes(st)))
        outs = [torch.full_like(k, 7) for _ in range(2)]
        B().relaxkv_read_quantized(st, i32([5, -1, bad, 5, -1, -1]), *outs, **kw)
        assert status() == B().ERR_BAD_INDEX
        for o in outs:
            assert (o[[1, 2, 4, 5]] == 7).all() and (o[[0, 3]] != 7).any(-1).all()
    changed = [(a != b).flatten(1).any(1) if a.dim() == 3 else (a != b).flatten(2).any(2) for a, b in zip(before, store_bytes(st))]
    assert changed[0].nonzero().tolist() == [[0, 5]]


# ---- reading ----

@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,Hkv,D,block,layout,pairs,part", [
    (1, 1, 64, 16, "token", "half", 64), (70, 8, 128, 16, "head", "interleaved", 128), (512, 8, 128, 64, "token", "half", 64), (1400, 8, 128, 32, "head", "half", 128),
    (3000, 2, 64, 128, "token", "interleaved", 24), (11, 5, 128, 16, "token", "half", 8)])
def test_rows_are_read(n, Hkv, D, block, layout, pairs, part, kind):
    n_blocks = n // block + 2
    st = make_store(n_blocks, block, Hkv, D, kind, layout)
    rng = np.random.default_rng(n)
    slots = rng.integers(0, n_blocks * block, n)                            # (a row may be read twice)
    kk, vv = (x[slots] for x in store_values(st))
    k, v = (laid_out(torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda"), layout) for _ in range(2))
    B().relaxkv_read_quantized(st, i32(slots), k, v)
    assert np.array_equal(f64(k), kk) and np.array_equal(f64(v), vv)
    pos, rot = rng.integers(-50000, 50000, n), rotary(part, pairs, 1.25)
    k2 = laid_out(torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda"), layout)
    B().relaxkv_read_quantized(st, i32(slots), k2, v, positions=i32(pos), rotary=rot)
    want = orc.turned(kk, None, 0, pos, rot.freq.cpu().numpy(), pairs == "interleaved", 1.25)
    assert (np.abs(f64(k2) - want) <= rotation_tolerance(kk, want, None, 1.25)).all() and np.array_equal(f64(v), vv)
    # what was read stands for the same when it is written again
    again = make_store(n // block + 1, block, Hkv, D, kind, layout, seed=9)
    B().relaxkv_append_quantized(again, k, v, i32(range(n)))
    for x, y in zip(store_values(again), (kk, vv)):
        assert np.array_equal(x[:n], y)
    assert status() == B().OK


# ---- attention ----

def attend(store, lens, new, H, block, seed=0, scale=None, width=None, q=None, gaps=False, ws=None, max_len=None, junk_pages=True):
    """lens: tokens of each sequence, new: rows of each that attend, the last ones (a list).  Returns what the call gave and what it should have."""
    rng = np.random.default_rng(seed)
    D, Hkv = store.dim, store.heads
    have = [-(-t // block) for t in lens]
    ids = rng.permutation(store.k.shape[0])[:sum(have)]
    width = width or max(max(have), 1)
    table = np.full((len(lens), width), 2 ** 31 - 1 if junk_pages else 0, dtype=np.int64)                   # behind a sequence's blocks: never looked at
    at = 0
    for i, h in enumerate(have):
        table[i, :h] = ids[at:at + h]
        at += h
    row_seq, row_len, cu = [], [], [0]
    for i, (t, n) in enumerate(zip(lens, new)):
        row_seq += [i] * n
        row_len += [max(0, t - n + 1 + j) for j in range(n)]
        cu.append(len(row_seq))
    n = len(row_seq)
    left = [r for r in range(n) if gaps and r % 3 == 1]
    seqs = [-1 if r in left else s for r, s in enumerate(row_seq)] + [-1] * 2                               # two rows behind the last sequence
    q = rnd(n + 2, H, D, seed=seed + 1) if q is None else q
    out, lse = torch.full((n + 2, H, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((H, n + 2), 7.0, device="cuda")
    rows = B().ContinuationRows([0, len(lens)], [n + 2], max(lens) if max_len is None else max_len, i32(cu), i32(seqs), i32(row_len + [0, 0]), i32(table))
    ws = workspace(H, Hkv, D) if ws is None else ws
    scale = D ** -0.5 if scale is None else scale
    run = lambda: B().relaxkv_quantized_attention(store, rows, q, out, ws, lse_out=lse, softmax_scale=scale)
    run()
    kk, vv = store_values(store)
    vs = value_scale(store)
    wants = []
    for i, t in enumerate(lens):
        slots = (table[i, :have[i], None] * block + np.arange(block)).reshape(-1)[:t].astype(int)
        r = slice(cu[i], cu[i + 1])
        wants.append(orc.attention(f64(q[r]), kk[slots], vv[slots], row_len[r], scale, vs[slots]))
    return dict(out=out, lse=lse, wants=wants, cu=cu, left=left, n=n, run=run, q=q, rows=rows, ws=ws, keep=(table,))


def check(r, D):
    out, lse = f64(r["out"]), f64(r["lse"])
    assert (out[r["n"]:] == 7).all() and (lse[:, r["n"]:] == 7).all()
    for (want, want_lse, *sizes), a, b in zip(r["wants"], r["cu"], r["cu"][1:]):
        tol, lse_tol = orc.attention_tolerance(want, want_lse, *sizes, D)
        for j, row in enumerate(range(a, b)):
            if row in r["left"]:
                assert (out[row] == 7).all() and (lse[:, row] == 7).all()
                continue
            assert (np.abs(out[row] - want[j]) <= tol[j]).all(), (row, np.abs(out[row] - want[j]).max(), tol[j].max())
            with np.errstate(invalid="ignore"):
                assert ((lse[:, row] == want_lse[:, j]) | (np.abs(lse[:, row] - want_lse[:, j]) <= lse_tol[:, j])).all(), (row, lse[:, row], want_lse[:, j])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("lens,new,H,Hkv,D,block,layout", [
    ([1], [1], 1, 1, 64, 16, "token"), ([0, 1, 15, 16, 17, 31, 32, 33], [1] * 8, 4, 1, 64, 16, "token"), ([64, 200, 0, 129, 513, 1000], [1, 2, 1, 3, 1, 8], 8, 2, 128, 16, "head"),
    ([700, 3], [33, 2], 5, 1, 128, 32, "token"), ([900] * 3, [1, 1, 1], 16, 1, 128, 64, "token"), ([333, 40], [7, 40], 32, 2, 64, 128, "head"),
    # longer than one block takes by itself
    ([5000], [1], 4, 1, 64, 16, "token"), ([3000, 17, 0, 9001, 1], [1, 1, 1, 1, 1], 32, 8, 128, 16, "token"), ([6000, 2500], [3, 5], 40, 8, 128, 64, "head"),
    ([4100, 1500], [20, 3], 10, 2, 128, 32, "token"), ([20000], [2], 16, 1, 128, 128, "token"), ([40000], [1], 3, 3, 64, 32, "head"), ([1, 1025], [1, 57], 8, 2, 128, 16, "token")])
def test_attention(lens, new, H, Hkv, D, block, layout, kind):
    store = make_store(sum(-(-t // block) for t in lens) + 3, block, Hkv, D, kind, layout, seed=len(lens))
    r = attend(store, lens, new, H, block, seed=3)
    check(r, D)
    out, lse = r["out"].clone(), r["lse"].clone()
    r["ws"].fill_(255)
    r["run"]()
    assert torch.equal(out, r["out"]) and torch.equal(lse, r["lse"]) and status() == B().OK              # the same bits again


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("lens", [[300, 70], [4000, 1100]])
def test_what_lies_behind_a_sequence_is_not_weighed(lens, kind):
    """The store is full of bytes and exponents of every kind; the tokens themselves are written over them."""
    Hkv, D, block = 2, 128, 64
    n = sum(-(-t // block) for t in lens)
    store = make_store(n, block, Hkv, D, kind, junk=True, seed=5)
    rng = np.random.default_rng(1)
    ids = np.random.default_rng(3).permutation(n)                           # (the blocks that attend() hands out)
    at = 0
    for t in lens:
        h = -(-t // block)
        slots = (ids[at:at + h, None] * block + np.arange(block)).reshape(-1)[:t]
        B().relaxkv_append_quantized(store, rnd(t, Hkv, D, seed=t), rnd(t, Hkv, D, seed=t + 1), i32(slots))
        at += h
    check(attend(store, lens, [2, 1], 8, block, seed=3), D)
    assert status() == B().OK


@pytest.mark.parametrize("lens,H,Hkv", [([50] * 130, 8, 2), ([1500] * 130, 2, 1), ([30] * 700, 4, 4)])
def test_many_sequences(lens, H, Hkv):
    lens = [max(0, t - 3 * i % t) for i, t in enumerate(lens)]
    lens[5] = 0
    store = make_store(sum(-(-t // 16) for t in lens), 16, Hkv, 64, "int8")
    check(attend(store, lens, [1 + (i % 5 == 2) for i in range(len(lens))], H, 16, seed=2, gaps=True), 64)
    assert status() == B().OK


@pytest.mark.parametrize("max_len", [None, 3000])
def test_rows_left_out_and_rows_that_contradict(max_len):
    """Row -1 within a tile; another sequence's row, a falling length: reported and left alone, the others are as they were."""
    Hkv, D, block, H = 2, 64, 16, 8
    store = make_store(60, block, Hkv, D, "int8")
    lens, new = [200, 300, 90], [6, 5, 7]
    r = attend(store, lens, new, H, block, gaps=True, max_len=max_len, width=200)
    check(r, D)
    assert status() == B().OK
    _, _, cu, seqs, row_len, table = r["rows"]._keep
    for name, row, value in (("seq", 8, 0), ("seq", 8, 3), ("seq", 8, -7), ("len", 8, 301), ("len", 8, -1)):
        s, l = seqs.clone(), row_len.clone()
        (s if name == "seq" else l)[row] = value
        rows = B().ContinuationRows([0, 3], [20], 3000 if max_len else 300, cu, s, l, table)
        out, lse = torch.full_like(r["out"], 7), torch.full_like(r["lse"], 7)
        B().relaxkv_quantized_attention(store, rows, r["q"], out, r["ws"], lse_out=lse, softmax_scale=D ** -0.5)
        assert status() == B().ERR_BAD_INDEX, (name, value)
        keep = [x for x in range(20) if x != 8]
        assert (out[8] == 7).all() and (lse[:, 8] == 7).all() and torch.equal(out[keep], r["out"][keep]) and torch.equal(lse[:, keep], r["lse"][:, keep])


@pytest.mark.parametrize("max_len", [None, 3000])
@pytest.mark.parametrize("what", ["last length beyond the table", "last length negative", "rows that fall", "rows beyond the call"])
def test_sequences_that_contradict(what, max_len):
    Hkv, D, block, H = 2, 64, 16, 8
    store = make_store(60, block, Hkv, D, "int8")
    r = attend(store, [200, 300, 90], [6, 5, 7], H, block, max_len=max_len)
    _, _, cu, seqs, row_len, table = r["rows"]._keep
    cu, row_len = cu.clone(), row_len.clone()
    gone = list(range(6, 11))
    if what == "last length beyond the table":
        row_len[10] = 19 * 16 + 1
    elif what == "last length negative":
        row_len[10] = -4
    elif what == "rows that fall":
        cu[2] = 5                                                           # sequence 1 has fewer than no rows, sequence 2 begins among the first's
        gone = list(range(5, 18))
    else:
        cu[3] = 21
        gone = list(range(11, 18))
    out, lse = torch.full_like(r["out"], 7), torch.full_like(r["lse"], 7)
    rows = B().ContinuationRows([0, 3], [20], 3000 if max_len else 400, cu, seqs, row_len, table)
    B().relaxkv_quantized_attention(store, rows, r["q"], out, r["ws"], lse_out=lse, softmax_scale=D ** -0.5)
    assert status() == B().ERR_BAD_INDEX
    keep = [x for x in range(20) if x not in gone]
    assert torch.equal(out[keep], r["out"][keep]) and torch.equal(lse[:, keep], r["lse"][:, keep])
    if what != "rows that fall":
        assert (out[gone] == 7).all() and (lse[:, gone] == 7).all()


@pytest.mark.parametrize("lens", [[100, 60], [3000, 1500]])
def test_blocks_that_are_none_are_passed_over(lens):
    Hkv, D, block, H = 2, 128, 32, 8
    store = make_store(200, block, Hkv, D, "e4m3")
    r = attend(store, lens, [2, 1], H, block)
    _, _, cu, seqs, row_len, table = r["rows"]._keep
    for bad in (-1, 200, 2 ** 31 - 1):
        t = table.clone()
        t[0, 1] = bad
        rows = B().ContinuationRows([0, 2], [5], max(lens), cu, seqs, row_len, t)
        B().relaxkv_quantized_attention(store, rows, r["q"], r["out"], r["ws"], lse_out=r["lse"])
        assert status() == B().ERR_BAD_INDEX
        kk, vv = store_values(store)
        slots = (r["keep"][0][0, :-(-lens[0] // block), None] * block + np.arange(block)).reshape(-1)[:lens[0]].astype(int)
        slots = np.delete(slots, np.arange(block, 2 * block))
        want = orc.attention(f64(r["q"][:2]), kk[slots], vv[slots], [lens[0] - 1 - block, lens[0] - block], D ** -0.5)
        check(dict(r, wants=[want, r["wants"][1]]), D)


def test_exponents_from_end_to_end():
    """Values of very different sizes beside each other, and keys and queries whose product alone is of ordinary size."""
    Hkv, D, block, H = 1, 64, 16, 4
    store = make_store(20, block, Hkv, D, "int8", seed=1)
    rng = np.random.default_rng(0)
    store.v_exp.copy_(torch.tensor(rng.integers(-100, 121, tuple(store.v_exp.shape)), dtype=torch.int8))
    check(attend(store, [250, 3], [2, 1], H, block), D)
    store.v_exp.copy_(torch.tensor(rng.integers(-100, -90, tuple(store.v_exp.shape)), dtype=torch.int8))
    check(attend(store, [250, 3], [2, 1], H, block), D)
    store.v_exp.fill_(-7)
    store.k_exp.fill_(100)
    check(attend(store, [250, 3], [2, 1], H, block, q=rnd(5, H, D, seed=4, scale=2.0 ** -105)), D)
    store.k_exp.fill_(-100)
    check(attend(store, [250, 3], [2, 1], H, block, q=rnd(5, H, D, seed=4, scale=2.0 ** 94)), D)
    assert status() == B().OK


@pytest.mark.parametrize("lens", [[40], [2000]])
def test_what_is_no_number_stays_with_its_rows(lens):
    """A NaN value reaches the outputs of the rows that see its token, a NaN key their lse too; a query that is no number only its own row and head."""
    Hkv, D, block, H = 1, 64, 16, 4
    store = make_store(lens[0] // 16 + 1, block, Hkv, D, "int8", seed=1)
    t = lens[0] - 1                                                         # of the last token only: row 1 sees it, row 0 does not
    r = attend(store, lens, [2], H, block)
    clean = r["out"].clone(), r["lse"].clone()
    x = int(r["keep"][0][0, t // 16])
    store.v_exp[x, 0, t % 16] = -128
    r["run"]()
    assert torch.equal(r["out"][0], clean[0][0]) and torch.isnan(r["out"][1]).all() and torch.equal(r["lse"], clean[1])
    store.k_exp[x, 0, t % 16] = -128
    r["run"]()
    assert torch.equal(r["out"][0], clean[0][0]) and torch.isnan(r["out"][1]).all() and torch.isnan(r["lse"][:, 1]).all() and torch.equal(r["lse"][:, 0], clean[1][:, 0])
    store.v_exp[x, 0, t % 16] = store.k_exp[x, 0, t % 16] = -8
    r["run"]()
    clean = r["out"].clone(), r["lse"].clone()
    r["q"][0, 2, 5], r["q"][1, 0, 0] = float("nan"), float("inf")
    r["run"]()
    bad = torch.zeros(4, H, dtype=torch.bool, device="cuda")
    bad[0, 2] = bad[1, 0] = True
    assert torch.isnan(r["out"][bad]).all() and torch.equal(r["out"][~bad], clean[0][~bad]) and torch.equal(r["lse"].t()[~bad], clean[1].t()[~bad])
    assert torch.isnan(r["lse"].t()[bad]).all() and status() == B().OK


def test_large_and_small_logits():
    """Weights that are one key's alone, and weights that are all alike."""
    Hkv, D, block, H = 2, 128, 16, 8
    for lens in ([700], [4000]):
        store = make_store(lens[0] // 16 + 1, block, Hkv, D, "int8", seed=1)
        for scale in (50.0, 1e-6):
            check(attend(store, lens, [2], H, block, scale=scale), D)
    assert status() == B().OK


def test_strides_of_a_store_within_a_larger_one():
    """Values in every other block and token of a larger tensor, K and V as they are laid out there."""
    Hkv, D, block, H = 2, 64, 16, 4
    base = [torch.randint(-127, 128, (80, 2 * block, 3, 2 * D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)).to(torch.int8) for i in range(2)]
    k, v = (x[::2, ::2, 1:, D:] for x in base)
    e = [torch.full((40, Hkv, block), -6, dtype=torch.int8, device="cuda") for _ in range(2)]
    store = B().QuantizedStore(k, v, *e)
    check(attend(store, [333, 100], [3, 1], H, block), D)
    before = [x.clone() for x in base]
    kk = rnd(5, Hkv, D, seed=1)
    B().relaxkv_append_quantized(store, kk, kk, i32([0, 17, 40, 639, 16]))
    assert np.array_equal(written(store, [0, 17, 40, 639, 16])[0][0], orc.quantized(f64(kk), "int8")[0])
    for x, y, z in zip(base, before, (k, v)):
        changed = x != y
        inside = torch.zeros_like(changed)
        inside[::2, ::2, 1:, D:] = True
        assert not (changed & ~inside).any()
    assert status() == B().OK


def test_graphs_and_streams_share_a_workspace():
    """Two captured calls of other shapes over one workspace, replayed in turn with other inputs and lengths, beside a call on a stream of its own."""
    Hkv, D, block, H = 2, 128, 16, 8
    store = make_store(700, block, Hkv, D, "int8")
    ws = workspace(H, Hkv, D)
    a, b = attend(store, [5000, 900], [1, 1], H, block, ws=ws, seed=1), attend(store, [3000], [9], H, block, ws=ws, seed=2)
    graphs = []
    for r in (a, b):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r["run"]()
        graphs.append(g)
    for r in (a, b):
        r["out"].fill_(7); r["lse"].fill_(7)
    ws.fill_(255)
    for g in graphs * 2:
        g.replay()
    check(a, D); check(b, D)
    # fewer tokens than captured, another query
    a["rows"]._keep[4].copy_(i32([1234, 0, 0, 0]))
    a["q"].copy_(rnd(4, H, D, seed=77))
    graphs[0].replay()
    kk, vv = store_values(store)
    slots = (a["keep"][0][0, :313, None] * block + np.arange(block)).reshape(-1)[:1234].astype(int)
    want = orc.attention(f64(a["q"][:1]), kk[slots], vv[slots], [1234], D ** -0.5)
    none = (np.zeros((1, H, D)), np.full((H, 1), -np.inf), np.zeros((1, H, D)), np.zeros((H, 1)), np.zeros((H, 1)))
    check(dict(a, wants=[want, none]), D)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = workspace(H, Hkv, D)
    out = torch.full_like(b["out"], 7)
    with torch.cuda.stream(side):
        B().relaxkv_quantized_attention(store, b["rows"], b["q"], out, other, lse_out=None, softmax_scale=D ** -0.5)
    graphs[0].replay()
    side.synchronize()
    assert torch.equal(out, b["out"]) and status() == B().OK


def test_a_step_as_it_is_used():
    """Chunks are put into the store, read back elsewhere, taken over as a context, continued by appended tokens, attended to."""
    Hkv, D, block, H, n = 2, 128, 16, 8, 160
    rot = rotary(64, "interleaved")
    chunks, ctx = make_store(20, block, Hkv, D, "int8", "head"), make_store(30, block, Hkv, D, "int8", seed=3)
    k, v = rnd(n, Hkv, D, seed=1), rnd(n, Hkv, D, seed=2)                   # encoded at positions 0 ..
    B().relaxkv_append_quantized(chunks, k, v, i32(range(n)))
    kc, vc = torch.empty_like(k), torch.empty_like(v)
    B().relaxkv_read_quantized(chunks, i32(range(n)), kc, vc, positions=torch.full((n,), 500, dtype=torch.int32, device="cuda"), rotary=rot)
    B().relaxkv_append_quantized(ctx, kc, vc, i32(range(n)))
    q, kn, vn = rnd(1, H, D, seed=4), rnd(1, Hkv, D, seed=5), rnd(1, Hkv, D, seed=6)
    B().relaxkv_append_quantized(ctx, kn, vn, i32([n]), q=q, positions=i32([500 + n]), rotary=rot)
    rows = B().ContinuationRows([0, 1], [1], n + 1, i32([0, 1]), i32([0]), i32([n + 1]), i32(np.arange(11)[None]))
    out = torch.empty_like(q)
    B().relaxkv_quantized_attention(ctx, rows, q, out, workspace(H, Hkv, D))
    kk, vv = (x[:n + 1] for x in store_values(ctx))
    want, lse, *sizes = orc.attention(f64(q), kk, vv, [n + 1], D ** -0.5)
    assert (np.abs(f64(out) - want) <= orc.attention_tolerance(want, lse, *sizes, D)[0]).all()
    # against the same in 64 bits without any rounding to 8: a key's or value's step is 2^-6 of its largest element at most, half of that is the error, twice for keys
    ang = lambda x, p: orc.turned(x, None, 0, p, rot.freq.cpu().numpy(), True, 1.0)
    full_k = np.concatenate([ang(f64(k), np.full(n, 500)), ang(f64(kn), [500 + n])])
    for x, y in ((kk, full_k), (vv, np.concatenate([f64(v), f64(vn)]))):
        assert (np.abs(x - y) <= (2.0 ** -7 * 2 + 2.0 ** -8) * 1.5 * np.abs(y).max(-1, keepdims=True) + 1e-6).all()
    assert status() == B().OK
