"""Attention over continuations with large values where tiles, pieces, blocks and lengths end, against a bound that one value row out of place
exceeds (tests/continuation_values.py)."""
import numpy as np
import pytest
import torch

from tests import continuation_values as val
from tests.test_gpu_continuations import ATTEND, B, SPARSE, Step, f64, get_bounds, status

pytestmark = pytest.mark.gpu


def edges(n, step):
    """0, n - 1 and both sides of every multiple of step."""
    at = np.unique(np.concatenate([[0, n - 1], np.arange(step, n, step) - 1, np.arange(step, n, step)]))
    return torch.from_numpy(at[(at >= 0) & (at < n)]).cuda()


def sharpen(s, step=64):
    for at, n in zip(s.at, s.ctx):
        if n > 0:
            s.v[at + edges(n, step)] *= 64
    last = {}
    for i, n in zip(s.row_seq, s.row_len):
        last[i] = max(n, last.get(i, 0))
    for i, n in last.items():
        for t in edges(n, 16).tolist() if n else []:
            s.vs[s.table[i][t // s.bs], t % s.bs] *= 64


def check(s, block=None, lists=None):
    s.k64, s.v64, s.ks64, s.vs64 = f64(s.k), f64(s.v), f64(s.ks), f64(s.vs)
    out, q, G = f64(s.out), f64(s.q), s.H // s.Hkv
    for r in range(len(s.row_seq)):
        for g in range(s.Hkv):
            heads = slice(g * G, (g + 1) * G)
            k, v = s.keys(r, g, block, lists)
            if len(k) == 0:
                assert (out[r, heads] == 0).all()
            else:
                assert val.check(out[r, heads], q[r, heads], k, v, float(np.float32(s.D ** -0.5))).all(), (r, g)


@pytest.mark.parametrize("name", [n for n in ATTEND if "large logits" not in n])
def test_shared_prefix_takes_every_value_once(name):
    s = Step(seed=200 + len(name), **ATTEND[name])
    sharpen(s)
    s.shared()
    assert status() == B().OK
    check(s)


@pytest.mark.parametrize("block,n_select", [(16, 9), (64, 7), (128, 3)])
@pytest.mark.parametrize("name", list(SPARSE))
def test_sparse_attention_takes_every_listed_value_once(name, block, n_select):
    b = B()
    s = Step(seed=300 + len(name) + block, **SPARSE[name])
    sharpen(s, 16)
    bounds, scale = get_bounds(s, block)
    lists = torch.full((len(s.row_seq), s.Hkv, n_select), -9, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, block, bounds, scale, s.rows(), s.q, 1, 1, lists, s.ws(block))
    s.sparse(block, lists)
    assert status() == b.OK
    check(s, block, lists.cpu().numpy())


@pytest.mark.parametrize("tokens", [1, 5, 17, 64, 127, 128, 129, 200])
def test_many_tokens_of_a_sequence_at_once(tokens):
    """A question of many tokens: each sees its sequence's own up to itself."""
    s = Step(8, 2, 128, [333, 0, 70], [1, 1, 2], [0, 30, 5, 0], [tokens, 2, 3, tokens], 16, seed=23)
    sharpen(s)
    s.shared()
    assert status() == B().OK
    check(s)
