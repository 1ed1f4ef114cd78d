"""The calls over contexts kept in 8 bits without a GPU: their oracle, the frequencies, and what the binding and the library refuse before any launch."""
import math

import numpy as np
import pytest
import torch

from paper_2609_33503_b200 import binding as B
from tests import quantized_oracle as orc


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


def store(n=4, block=16, heads=2, dim=64, dtype=torch.int8):
    return B.QuantizedStore.empty(n, block, heads, dim, dtype, "cpu")


def rotary(dims=64, **kw):
    return B.Rotary(torch.ones(dims // 2, dtype=torch.float64), **kw)


# ---- the oracle against torch's conversions ----

def test_oracle_rounds_like_the_type():
    x = torch.randn(400, 1, 64, generator=torch.Generator().manual_seed(1)).double() * torch.logspace(-3, 2, 64).double()
    x[:40] = torch.randint(-64, 64, (40, 1, 64), generator=torch.Generator().manual_seed(2)).double() / 16          # ties
    for kind, dtype in (("int8", torch.int8), ("e4m3", torch.float8_e4m3fn)):
        v, e = orc.quantized(x.numpy(), kind)
        y = torch.ldexp(x, -torch.tensor(e)[..., None])
        assert (y.abs() <= orc.MOST[kind]).all() and (2 * y.abs().amax(-1) > orc.MOST[kind]).all()
        want = torch.round(y) if kind == "int8" else y.float().to(dtype).double()
        assert np.array_equal(v, want.numpy())


def test_oracle_attention_is_a_softmax():
    g = np.random.default_rng(3)
    q, k, v = g.normal(size=(3, 4, 8)), g.normal(size=(9, 2, 8)), g.normal(size=(9, 2, 8))
    out, lse, *_ = orc.attention(q, k, v, [9, 0, 4], 0.5)
    kk, vv = torch.tensor(k).repeat_interleave(2, 1)[:4], torch.tensor(v).repeat_interleave(2, 1)[:4]
    s = torch.einsum("hd,thd->ht", torch.tensor(q[2]), kk) * 0.5
    assert np.allclose(out[2], torch.einsum("ht,thd->hd", s.softmax(-1), vv).numpy()) and np.allclose(lse[:, 2], s.logsumexp(-1).numpy())
    assert (out[1] == 0).all() and (lse[:, 1] == -np.inf).all()


def test_oracle_rotation_is_a_product_of_complex_numbers():
    x = np.random.default_rng(4).normal(size=(5, 2, 16))
    freq, pos = np.array([1.0, 0.3, 0.01, 0.002]), np.arange(5) * 7 - 9
    for inter in (False, True):
        y = orc.turned(x, None, 0, pos, freq, inter, 1.5)
        a, b = (np.s_[..., 0:8:2], np.s_[..., 1:8:2]) if inter else (np.s_[..., :4], np.s_[..., 4:8])
        z = (x[a] + 1j * x[b]) * 1.5 * np.exp(1j * pos[:, None, None] * freq)
        assert np.allclose(y[a], z.real) and np.allclose(y[b], z.imag) and np.array_equal(y[..., 8:], x[..., 8:])


# ---- frequencies ----

def test_frequencies():
    freq, amp = B.relaxkv_rotary_frequencies(128, 5e5)
    assert amp == 1 and np.allclose(freq, [5e5 ** (-2 * i / 128) for i in range(64)], rtol=1e-14)
    half, amp = B.relaxkv_rotary_frequencies(64, 1e4, "linear", 4.0)
    assert amp == 1 and np.allclose(half, [1e4 ** (-2 * i / 64) / 4 for i in range(32)], rtol=1e-14)


def test_frequencies_in_bands():
    plain, _ = B.relaxkv_rotary_frequencies(128, 5e5)
    freq, amp = B.relaxkv_rotary_frequencies(128, 5e5, "bands", 8.0, 8192, 1.0, 4.0)
    turns = [8192 * f / (2 * math.pi) for f in plain]
    assert amp == 1 and any(1 < t < 4 for t in turns)
    for f, p, t in zip(freq, plain, turns):
        if t >= 4:
            assert f == p
        elif t <= 1:
            assert abs(f - p / 8) <= 1e-15 * p
        else:
            s = (t - 1) / 3
            assert abs(f - (s * p + (1 - s) * p / 8)) <= 1e-14 * p


def test_frequencies_by_a_ramp():
    plain, _ = B.relaxkv_rotary_frequencies(128, 1e6)
    freq, amp = B.relaxkv_rotary_frequencies(128, 1e6, "ramp", 4.0, 32768, 1.0, 32.0)
    assert abs(amp - (0.1 * math.log(4) + 1)) < 1e-6
    share = [(p / f - 1) / 3 for f, p in zip(freq, plain)]                 # 0: as it was; 1: a quarter of it
    assert share[0] == 0 and abs(share[-1] - 1) < 1e-12 and all(b >= a - 1e-12 for a, b in zip(share, share[1:]))
    lo = math.floor(128 * math.log(32768 / (2 * math.pi * 32)) / (2 * math.log(1e6)))
    hi = math.ceil(128 * math.log(32768 / (2 * math.pi)) / (2 * math.log(1e6)))
    for i, (f, p) in enumerate(zip(freq, plain)):
        r = min(1, max(0, (i - lo) / (hi - lo)))
        assert abs(f - p * (1 - r + r / 4)) <= 1e-14 * p
    same, amp = B.relaxkv_rotary_frequencies(128, 1e6, "ramp", 1.0, 32768, 1.0, 32.0)
    assert amp == 1 and np.allclose(same, plain, rtol=1e-14)


@pytest.mark.parametrize("args", [(0, 1e4), (12, 1e4), (64, 1.0), (64, float("nan")), (64, 1e4, "linear", 0.5), (64, 1e4, "bands", 2.0, 0, 1.0, 4.0),
                                  (64, 1e4, "bands", 2.0, 100, 4.0, 4.0), (64, 1e4, "ramp", 2.0, 100, 0.0, 4.0), (64, 1e4, "ramp", float("inf"), 100, 1.0, 4.0)])
def test_frequencies_refused(args):
    with pytest.raises(B.RelaxKVError):
        B.relaxkv_rotary_frequencies(*args)


# ---- what the binding refuses ----

def test_rotate_marshals_and_refuses(calls):
    fused = bf(5, 6, 64)                                                   # a row's heads of q, k and v side by side
    q, k = fused[:, :3], fused[:, 3:4]
    B.relaxkv_qk_norm_rotate(q, k, i32(5), rotary(), stream=0)
    name, a = calls.pop()
    assert name == "relaxkv_qk_norm_rotate" and len(a) == 18 and a[:4] == (q.data_ptr(), q.data_ptr(), 384, 64) and a[4:8] == (k.data_ptr(), k.data_ptr(), 384, 64)
    assert a[8:12] == (5, 3, 1, 64)
    B.relaxkv_qk_norm_rotate(None, k, i32(5), rotary(), k_out=torch.empty_strided(k.shape, k.stride(), dtype=k.dtype), stream=0)
    assert calls.pop()[1][:4] == (None, None, 0, 0)
    bad = [dict(q=None, k=None), dict(positions=i32(4)), dict(positions=torch.zeros(5, dtype=torch.int64)), dict(k=bf(4, 1, 64)), dict(k=bf(5, 1, 128)),
           dict(q=q.float()), dict(q_out=bf(5, 3, 64)), dict(k_out=bf(5, 2, 64)), dict(q=bf(5, 64, 3).transpose(1, 2)), dict(w_q_norm=bf(63), w_k_norm=bf(64)),
           dict(w_q_norm=torch.zeros(64), w_k_norm=bf(64)), dict(q=bf(5, 64))]
    for kw in bad:
        args = dict(q=q, k=k, positions=i32(5), rotary=rotary())
        with pytest.raises(ValueError):
            B.relaxkv_qk_norm_rotate(**dict(args, **kw), stream=0)
    assert not calls


def test_append_marshals_and_refuses(calls):
    args = dict(store=store(), k=bf(7, 2, 64), v=bf(7, 2, 64), slots=i32(7))
    B.relaxkv_append_quantized(**args, stream=0)
    name, a = calls.pop()
    assert name == "relaxkv_append_quantized" and len(a) == 20 and a[1:5] == (None, None, 0, 0) and a[7:13] == (128, 64, 7, 0, 2, 64) and a[16] is None and a[17] is None
    q = bf(7, 8, 64)
    B.relaxkv_append_quantized(**args, q=q, positions=i32(7), rotary=rotary(), stream=0)
    assert calls.pop()[1][1:5] == (q.data_ptr(), q.data_ptr(), 512, 64)
    for kw in (dict(slots=i32(6)), dict(slots=torch.zeros(7, dtype=torch.int64)), dict(k=bf(7, 3, 64), v=bf(7, 3, 64)), dict(k=bf(7, 2, 128), v=bf(7, 2, 128)), dict(v=bf(6, 2, 64)),
               dict(v=bf(2, 7, 64).transpose(0, 1)), dict(v=torch.zeros(7, 2, 64)), dict(q=bf(6, 8, 64)), dict(q=bf(7, 8, 128)), dict(q_out=bf(7, 8, 64)),
               dict(positions=i32(3), rotary=rotary()), dict(q=q, q_out=bf(7, 4, 64))):
        with pytest.raises(ValueError):
            B.relaxkv_append_quantized(**dict(args, **kw), stream=0)
    assert not calls


def test_read_marshals_and_refuses(calls):
    out = bf(2, 9, 64).transpose(0, 1)                                     # head-major
    args = dict(store=store(), slots=i32(9), k_out=out, v_out=bf(2, 9, 64).transpose(0, 1))
    B.relaxkv_read_quantized(**args, stream=0)
    name, a = calls.pop()
    assert name == "relaxkv_read_quantized" and len(a) == 12 and a[2:7] == (9, 2, 64, None, None) and a[9:11] == (64, 576)
    for kw in (dict(slots=i32(8)), dict(k_out=bf(9, 2, 64)), dict(k_out=bf(9, 3, 64), v_out=bf(9, 3, 64)), dict(v_out=torch.zeros(9, 2, 64)), dict(positions=i32(8), rotary=rotary())):
        with pytest.raises(ValueError):
            B.relaxkv_read_quantized(**dict(args, **kw), stream=0)
    assert not calls


def rows(n=6, n_seq=3, width=5, max_len=70):
    return B.ContinuationRows([0, n_seq], [n], max_len, i32(n_seq + 1), i32(n), i32(n), i32(n_seq, width))


def test_attention_marshals_and_refuses(calls):
    args = dict(store=store(), rows=rows(), q=bf(6, 8, 64), out=bf(6, 8, 64), workspace=torch.zeros(512, dtype=torch.uint8))
    B.relaxkv_quantized_attention(**args, stream=0)
    name, a = calls.pop()
    assert name == "relaxkv_quantized_attention" and len(a) == 12 and a[2:6] == (8, 2, 64, 0.125) and a[8] is None and a[10] == 512
    for kw in (dict(q=bf(5, 8, 64)), dict(q=bf(6, 8, 128)), dict(out=bf(6, 7, 64)), dict(q=bf(6, 64, 8).transpose(1, 2)), dict(q=torch.zeros(6, 8, 64)),
               dict(lse_out=torch.zeros(47)), dict(lse_out=bf(8, 6))):
        with pytest.raises(ValueError):
            B.relaxkv_quantized_attention(**dict(args, **kw), stream=0)
    assert not calls


@pytest.mark.parametrize("what", ["scales of another shape", "of another type", "values of bf16", "k and v apart", "dims apart"])
def test_a_store_is_what_it_says(what):
    k, v, e = (torch.zeros(4, 16, 2, 64, dtype=torch.int8) for _ in range(2)), None, torch.zeros(4, 2, 16, dtype=torch.int8)
    k, v = k
    f = e.clone()
    if what == "scales of another shape":
        f = torch.zeros(4, 16, 2, dtype=torch.int8)
    elif what == "of another type":
        f = torch.zeros(4, 2, 16)
    elif what == "values of bf16":
        k = v = bf(4, 16, 2, 64)
    elif what == "k and v apart":
        v = v.transpose(1, 2).contiguous().transpose(1, 2)
    else:
        k = v = torch.zeros(4, 16, 64, 2, dtype=torch.int8).transpose(2, 3)
    with pytest.raises(AssertionError):
        B.QuantizedStore(k, v, e, f)


# ---- what the library refuses (addresses that nothing is read from: every check stands before the first launch) ----

P = 1 << 20                                                                # an aligned address


def c_store(**kw):
    a = dict(k=P, v=P, k_exp=P, v_exp=P, block_stride=16 * 128, token_stride=128, head_stride=64, block_size=16, n_blocks=4, n_kv_heads=2, type=0)
    a.update(kw)
    return B._QuantizedCache(*[a[n] for n, _ in B._QuantizedCache._fields_])


def c_rotary(**kw):
    a = dict(freq=P, dims=64, interleaved=0, amplitude=1.0)
    a.update(kw)
    return B._Rotary(*[a[n] for n, _ in B._Rotary._fields_])


BAD_STORES = [dict(k=0), dict(v=P + 8), dict(k_exp=0), dict(v_exp=P + 1), dict(type=2), dict(type=-1), dict(block_size=24), dict(block_size=256), dict(n_blocks=0),
              dict(n_blocks=1 << 28), dict(token_stride=72), dict(block_stride=48), dict(head_stride=32), dict(n_kv_heads=3), dict(n_kv_heads=0)]
BAD_ROTARIES = [dict(freq=0), dict(freq=P + 4), dict(dims=12), dict(dims=72), dict(dims=-8), dict(interleaved=2), dict(amplitude=0.0), dict(amplitude=float("nan")),
                dict(amplitude=float("inf"))]


def call(name, codes, *args):
    return getattr(B.lib(), name)(*B._args(codes, *args))


def rotate_c(rot=None, q=P, q_out=P, qt=512, qh=64, k=P, k_out=P, kt=128, kh=64, n=3, H=8, Hkv=2, D=64, wq=None, wk=None, eps=1e-6, pos=P):
    return call("relaxkv_qk_norm_rotate", "................s.", q, q_out, qt, qh, k, k_out, kt, kh, n, H, Hkv, D, wq, wk, eps, pos, rot or c_rotary(), 0)


def append_c(st=None, rot=None, q=None, q_out=None, qt=512, qh=64, k=P, v=P, kt=128, kh=64, n=3, H=8, Hkv=2, D=64, wq=None, wk=None, eps=1e-6, pos=None, slots=P):
    return call("relaxkv_append_quantized", "s................" + ("s" if rot else ".") + "..", st or c_store(), q, q_out, qt, qh, k, v, kt, kh, n, H, Hkv, D, wq, wk, eps, pos,
                rot, slots, 0)


def read_c(st=None, rot=None, slots=P, n=3, Hkv=2, D=64, pos=None, k=P, v=P, ts=128, hs=64):
    return call("relaxkv_read_quantized", "s....." + ("s" if rot else ".") + ".....", st or c_store(), slots, n, Hkv, D, pos, rot, k, v, ts, hs, 0)


def attend_c(st=None, H=8, Hkv=2, D=64, scale=0.1, q=P, out=2 * P, ws=P, nbytes=1 << 30, **kw):
    a = dict(n_seq=3, table_width=5, table_stride=5, n_rows=6, max_len=70, h_seq_cu=None, h_max_rows=None, row_cu=P, row_seq=P, row_len=P, block_table=P)
    a.update(kw)
    r = B._ContinuationRows(*[a[n] for n, _ in B._ContinuationRows._fields_])
    return call("relaxkv_quantized_attention", "ss..........", st or c_store(), r, H, Hkv, D, scale, q, out, None, ws, nbytes, 0)


REFUSED = (B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED_SHAPE, B.ERR_WORKSPACE_TOO_SMALL)


def test_calls_of_no_rows_are_taken():
    assert rotate_c(n=0) == append_c(n=0) == read_c(n=0) == attend_c(n_rows=0) == B.OK


@pytest.mark.parametrize("kw", BAD_STORES)
def test_library_refuses_stores(kw):
    st = c_store(**kw)
    for f in (append_c, read_c, attend_c):
        assert f(st, **({"n_rows": 0} if f is attend_c else {"n": 0})) in REFUSED


@pytest.mark.parametrize("kw", BAD_ROTARIES)
def test_library_refuses_rotaries(kw):
    rot = c_rotary(**kw)
    assert rotate_c(rot, n=0) in REFUSED and append_c(rot=rot, pos=P, n=0) in REFUSED and read_c(rot=rot, pos=P, n=0) in REFUSED


@pytest.mark.parametrize("f,kw", [(rotate_c, kw) for kw in (dict(q=None, q_out=None, k=None, k_out=None), dict(q_out=None), dict(k=None), dict(q=P + 8), dict(qt=500), dict(qh=60),
                                                            dict(kt=32), dict(kh=72 + 4), dict(n=-1), dict(n=1 << 31), dict(H=0), dict(Hkv=0), dict(D=96), dict(wq=P),
                                                            dict(eps=-1.0), dict(eps=float("nan")), dict(pos=None))]
                         + [(append_c, kw) for kw in (dict(slots=None), dict(q=P), dict(q_out=P), dict(k=None), dict(v=None), dict(v=P + 2), dict(kt=60), dict(kh=12), dict(n=-1), dict(Hkv=4),
                                                      dict(D=128), dict(wk=P), dict(eps=-1.0), dict(rot=c_rotary()), dict(q=P, q_out=P, H=0))]
                         + [(read_c, kw) for kw in (dict(slots=None), dict(n=-1), dict(Hkv=1), dict(D=32), dict(pos=P), dict(rot=c_rotary()), dict(k=None), dict(v=P + 8), dict(ts=8), dict(hs=68))]
                         + [(attend_c, kw) for kw in (dict(H=7), dict(H=64), dict(Hkv=0), dict(D=96), dict(scale=0.0), dict(scale=float("nan")), dict(q=None), dict(out=None), dict(out=P),
                                                      dict(q=P + 2), dict(ws=None), dict(ws=P + 128), dict(nbytes=1000), dict(n_seq=0), dict(n_seq=4097), dict(n_rows=-1), dict(n_rows=1 << 31),
                                                      dict(max_len=-1), dict(max_len=0x7fffff01), dict(row_cu=None), dict(row_seq=None), dict(row_len=None), dict(block_table=None),
                                                      dict(table_width=0), dict(table_stride=4))])
def test_library_refuses_arguments(f, kw):
    none = {"n_rows": 0} if f is attend_c else {"n": 0}
    assert f(**dict(none, **kw)) in REFUSED


def test_workspace_bytes():
    n = B.relaxkv_quantized_workspace_bytes(40, 8, 128)
    assert n == B.relaxkv_quantized_workspace_bytes(8, 8, 128) > 0 and n % 256 == 0
    for bad in ((40, 7, 128), (0, 1, 128), (34, 2, 128), (8, 8, 96)):
        assert B.relaxkv_quantized_workspace_bytes(*bad) == 0
    assert attend_c(D=64, nbytes=B.relaxkv_quantized_workspace_bytes(8, 2, 64), n_rows=0) == B.OK
