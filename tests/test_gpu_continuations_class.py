"""Continuations (paper_2609_33503_b200.continuations) against the framework's own query pass, which runs one continuation of each context over
the contiguous cache, and against itself."""
import pytest
import torch

from paper_2609_33503_b200 import inputs

pytestmark = pytest.mark.gpu

H, HKV, D, L = 8, 2, 128, 2
BLK = inputs.BlockShape(hidden=512, inter=1024, rope_theta=1.0e4, eps=1.0e-5, qk_norm=True)


def B():
    from paper_2609_33503_b200 import binding
    return binding


def rnd(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)


def setup(ctx, extra):
    w = inputs.Workload("continuations", L, H, HKV, D, 64, tuple(ctx), (1,) * len(ctx), 0.15, base_seed=3, planted_chunks=((0,),) * len(ctx))
    weights = [inputs.block_weights(w, BLK, l, "cuda") for l in range(L)]
    room = [t + extra for t in ctx]
    at = [sum(room[:b]) for b in range(len(ctx))]
    caches = [B().CacheView(rnd(sum(room), HKV, D, seed=10 + l), rnd(sum(room), HKV, D, seed=20 + l), at) for l in range(L)]
    return weights, caches


def status():
    torch.cuda.synchronize()
    return B().relaxkv_read_device_status()[0]


def same(a, b):
    """Two layers of bf16 arithmetic in another order: each is some 8e-3 of the exact rows away (chains of 6 to 12 layers 8e-3 to 1.3e-2)."""
    a, b = a.double(), b.double()
    return float((a - b).norm() / b.norm()) <= 1.6e-2


@pytest.mark.parametrize("n_select", [0, 64])
def test_question_and_answers_match_the_query_pass(n_select):
    """A question of several tokens and three decoded ones per context; with 64 selected blocks of 16 every context is read whole."""
    from paper_2609_33503_b200.continuations import Continuations
    from paper_2609_33503_b200.query_pass import QueryPass
    ctx, qn = (700, 301), (9, 4)
    weights, caches = setup(ctx, 16)
    qp = QueryPass(H, HKV, D, ctx, qn, BLK, extra_tokens=4)
    c = Continuations(H, HKV, D, ctx, (1, 1), L, BLK, n_blocks=6, max_len=40, block_size=16, max_rows=16, n_select=n_select, ctx_block=16)
    c.context_bounds(caches)
    x = rnd(sum(qn), BLK.hidden, seed=1)
    want = qp.prefill(x, weights, caches).clone()
    assert c.begin(qn) == sum(qn)
    assert same(c.run(x, weights, caches), want)
    for step in range(3):
        x = rnd(2, BLK.hidden, seed=2 + step)
        want = qp.decode(x, weights, caches, step=step).clone()
        assert c.begin((1, 1)) == 2
        got = c.run(x, weights, caches)
        assert same(got, want)
    logits = torch.empty(2, 104, dtype=torch.bfloat16, device="cuda")
    c.output_head(got, rnd(BLK.hidden, seed=8), rnd(104, BLK.hidden, seed=9), logits)
    assert torch.isfinite(logits).all() and status() == B().OK
    assert c.lens == [q + 3 for q in qn] == c._len[0].tolist() and c._n_free[0].tolist() == [c.n_free]


def test_a_step_of_fewer_rows_fits_the_room_of_the_largest():
    """Steps of every size that the object was made for, on a stream of their own as well."""
    from paper_2609_33503_b200.continuations import Continuations
    ctx = (200,)
    weights, caches = setup(ctx, 0)
    c = Continuations(H, HKV, D, ctx, (1,), L, BLK, n_blocks=16, max_len=256, block_size=16, max_rows=100)
    for n in (100, 1, 64):
        x = rnd(n, BLK.hidden, seed=n)
        c.begin([-1])
        assert c.begin([n]) == n
        want = c.run(x, weights, caches).clone()
        c.begin([-1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            assert c.begin([n]) == n
            got = c.run(x, weights, caches)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got, want) and status() == B().OK


def test_samples_do_not_disturb_each_other():
    """Four samples of two contexts: the same tokens give the same rows whatever the others do, through ends, waits and blocks used again."""
    from paper_2609_33503_b200.continuations import Continuations
    ctx = (260, 90)
    weights, caches = setup(ctx, 0)
    make = lambda seqs, n: Continuations(H, HKV, D, ctx, seqs, L, BLK, n_blocks=n, max_len=64, block_size=16, max_rows=12)
    alone, many = make((1, 0), 4), make((2, 2), 9)
    steps = [([3, 20, 1, 5], 3), ([1, 1, 0, 1], 1), ([1, -1, 1, 1], 1), ([1, 14, 1, 1], 1), ([1, 1, -1, 1], 1)]
    for i, (new, mine) in enumerate(steps):
        rows = sum(n for n in new if n > 0)
        if rows > many.max_rows:
            with pytest.raises(ValueError, match="rows"):
                many.begin(new)
            new = [new[0], 3, new[2], new[3]]
            rows = sum(new)
        assert many.begin(new) == rows and alone.begin([mine]) == mine
        x = rnd(rows, BLK.hidden, seed=50 + i)
        a, b = alone.run(x[:mine], weights, caches).clone(), many.run(x, weights, caches)
        assert same(b[:mine], a), i
        assert many._len[0].tolist() == many.lens and many._n_free[0].tolist() == [many.n_free]
        held = [many.table[s, :-(-t // 16)].tolist() for s, t in enumerate(many.lens)]
        free = many.free[:many.n_free].tolist()
        assert sorted(sum(held, []) + free) == list(range(9))            # every block once
    with pytest.raises(ValueError, match="blocks short"):
        make((2, 0), 1).begin([4, 1])
    with pytest.raises(ValueError, match="room for"):
        c = Continuations(H, HKV, D, ctx, (1, 0), L, BLK, n_blocks=9, max_len=16, block_size=16, max_rows=40)
        c.begin([17])
    with pytest.raises(ValueError):
        many.begin([1, 1])
    assert status() == B().OK


def test_a_step_of_nothing():
    from paper_2609_33503_b200.continuations import Continuations
    weights, caches = setup((64,), 0)
    c = Continuations(H, HKV, D, (64,), (2,), L, BLK, n_blocks=2, max_len=16, block_size=16)
    assert c.begin([0, 0]) == 0
    x = torch.empty(0, BLK.hidden, dtype=torch.bfloat16, device="cuda")
    assert c.run(x, weights, caches).shape[0] == 0
    assert c.begin([1, 0]) == 1 and c.begin([-1, -1]) == 0 and c.n_free == 2
    assert status() == B().OK


def test_the_example_runs():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "sample_answers.py"), "--ctx", "2048", "--layers", "2", "--samples", "4", "--steps", "3"],
                       capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "4 samples" in r.stdout
