"""One token's heads, cut from a fused projection, through the calls over rows of heads: the same bits as rows by themselves give."""
import pytest
import torch

from tests.test_gpu_quantized import B, i32, make_store, rnd, rotary, status, store_bytes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv", [(8, 2), (4, 1), (1, 1)])
def test_one_row_of_a_fused_projection(H, Hkv):
    D = 64
    fused = rnd(3, (H + 2 * Hkv) * D, seed=1).unflatten(1, (-1, D))[1:2]
    q, k, v = fused[:, :H], fused[:, H:H + Hkv], fused[:, H + Hkv:]
    own = [x.contiguous() for x in (q, k, v)]
    pos, rot = i32([1234]), rotary(48, "half")
    a, b = [torch.empty(1, n, D, dtype=torch.bfloat16, device="cuda") for n in (H, Hkv)], [torch.empty(1, n, D, dtype=torch.bfloat16, device="cuda") for n in (H, Hkv)]
    B().relaxkv_qk_norm_rotate(q, k, pos, rot, *a)
    B().relaxkv_qk_norm_rotate(own[0], own[1], pos, rot, *b)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    stores = [make_store(2, 16, Hkv, D, "int8", seed=2) for _ in range(2)]
    B().relaxkv_append_quantized(stores[0], k, own[2], i32([7]), q=q, q_out=a[0], positions=pos, rotary=rot)
    B().relaxkv_append_quantized(stores[1], own[1], own[2], i32([7]), q=own[0], q_out=b[0], positions=pos, rotary=rot)
    assert torch.equal(a[0], b[0]) and all(torch.equal(x, y) for x, y in zip(*(store_bytes(s) for s in stores)))
    room = torch.zeros(4, Hkv + 1, D, dtype=torch.bfloat16, device="cuda")
    out = [torch.empty(1, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B().relaxkv_read_quantized(stores[0], i32([7]), *out, positions=pos, rotary=rot)
    B().relaxkv_read_quantized(stores[0], i32([7]), room[2:3, 1:], torch.empty_like(out[1]), positions=pos, rotary=rot)
    assert torch.equal(room[2:3, 1:], out[0]) and (room[[0, 1, 3]] == 0).all() and (room[2, 0] == 0).all() and status() == B().OK
