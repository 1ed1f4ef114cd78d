"""Rows of the 8-bit store read back over the whole range of their exponents, -100 to 127."""
import numpy as np
import pytest
import torch

from tests import quantized_oracle as orc
from tests.test_gpu_quantized import B, TYPES, f64, i32, make_store, rotary, rotation_tolerance, status, store_values

pytestmark = pytest.mark.gpu


def as_bf16(x):
    """What a value times a power of two is in bf16: itself, or infinite from 2^128 on."""
    return np.where(np.abs(x) >= 2.0 ** 128, np.sign(x) * np.inf, x)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("Hkv,D,layout", [(1, 64, "token"), (3, 128, "head")])
def test_rows_are_read_at_every_exponent(kind, Hkv, D, layout):
    """As they are: exact, whatever the exponent; no element of a row has anything to do with the others."""
    n_blocks, block = 16, 16
    st = make_store(n_blocks, block, Hkv, D, kind, layout, seed=1)
    n = n_blocks * block
    e = torch.arange(n, device="cuda").clamp(max=227).sub(100).to(torch.int8).reshape(n_blocks, 1, block).expand(n_blocks, Hkv, block)
    st.k_exp.copy_(e)
    st.v_exp.copy_(e.flip(0))
    st.k.view(torch.int8)[:, :, 0, :2] = 0                                  # zeros among them
    kk, vv = store_values(st)
    k, v = (torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B().relaxkv_read_quantized(st, i32(range(n)), k, v)
    assert np.array_equal(f64(k), as_bf16(kk)) and np.array_equal(f64(v), as_bf16(vv)) and status() == B().OK


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("pairs", ["half", "interleaved"])
def test_rows_are_turned_at_every_exponent(kind, pairs):
    """Turned: up to exponents at which no sum of a pair's products leaves fp32 (values to 448, a pair to 1.5 times the larger)."""
    n_blocks, block, Hkv, D = 14, 16, 2, 64
    st = make_store(n_blocks, block, Hkv, D, kind, seed=2)
    n, most = n_blocks * block, 117
    e = torch.arange(n, device="cuda").clamp(max=most + 100).sub(100).to(torch.int8).reshape(n_blocks, 1, block).expand(n_blocks, Hkv, block)
    st.k_exp.copy_(e)
    st.v_exp.copy_(e)
    kk, vv = store_values(st)
    k, v = (torch.empty(n, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, rot = np.random.default_rng(3).integers(-50000, 50000, n), rotary(48, pairs)
    B().relaxkv_read_quantized(st, i32(range(n)), k, v, positions=i32(pos), rotary=rot)
    want = orc.turned(kk, None, 0, pos, rot.freq.cpu().numpy(), pairs == "interleaved", 1.0)
    assert (np.abs(f64(k) - want) <= rotation_tolerance(kk, want, None, 1.0)).all() and np.array_equal(f64(v), vv) and status() == B().OK


@pytest.mark.parametrize("kind", list(TYPES))
def test_large_elements_come_back(kind):
    """Heads of elements up to bf16's largest: appended, read, appended again.  An element that the rounding to 8 bits takes to 2^128 comes back infinite; all others as the store has them."""
    n, Hkv, D, block = 30, 2, 128, 16
    x = torch.randn(n, Hkv, D, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").clamp(-3.9, 3.9)
    k = (x * torch.exp2(torch.arange(n, device="cuda").float() + 97)[:, None, None]).to(torch.bfloat16)     # up to 3.9 * 2^126
    k[-1, 0, 0], k[-1, 0, 1] = torch.finfo(torch.bfloat16).max, 1.0
    assert torch.isfinite(k).all()
    st, again = (B().QuantizedStore.empty(2, block, Hkv, D, TYPES[kind]) for _ in range(2))
    B().relaxkv_append_quantized(st, k, k, i32(range(n)))
    values, e = orc.quantized(f64(k), kind)
    want = as_bf16(orc.values(values, e))
    out = [torch.empty_like(k) for _ in range(2)]
    B().relaxkv_read_quantized(st, i32(range(n)), *out)
    assert all(np.array_equal(f64(o), want) for o in out)
    B().relaxkv_append_quantized(again, *out, i32(range(n)))
    finite = np.isfinite(want).all(-1)
    assert finite.sum() >= 2 * n - 2
    for got in store_values(again):
        assert np.array_equal(got[:n][finite], want[finite]) and np.isnan(got[:n][~finite]).all()
    assert status() == B().OK
