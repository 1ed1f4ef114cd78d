"""Continuations on the GPU over ranges that meet in one call: contexts of very different length, logits and values of very different size."""
import numpy as np
import pytest
import torch

from tests import continuation_oracle as orc
from tests.test_gpu_continuations import B, Step, f64, get_bounds, i32, status

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ctx", [(140000, 3000), (3000, 140000), (300, 131200, 0, 140000, 9000)])
@pytest.mark.parametrize("n_select,n_first,n_last", [(9, 1, 2), (200, 0, 3), (3, 1, 2)])
def test_selection_in_contexts_beside_one_of_very_many_blocks(ctx, n_select, n_first, n_last):
    """140000 tokens in blocks of 16: more blocks than the selection keeps the scores of, beside contexts of fewer."""
    b = B()
    s = Step(2, 1, 64, list(ctx), [2] * len(ctx), 3, 1, 16, seed=21)
    bounds, scale = get_bounds(s, 16)
    n = len(s.row_seq)
    lists = torch.full((n, 1, n_select), -9, dtype=torch.int32, device="cuda")
    b.relaxkv_select_blocks(s.shape, 16, bounds, scale, s.rows(), s.q, n_first, n_last, lists, s.ws(16))
    assert status() == b.OK
    at = np.concatenate([[0], np.cumsum([-(-t // 16) for t in ctx])])
    bi, sc, q = bounds.cpu().numpy().astype(np.int64), f64(scale), f64(s.q)
    for r in range(n):
        c = s.context_of(r)
        want = orc.select(q[r], bi[at[c]:at[c + 1]], sc[at[c]:at[c + 1]], n_select, n_first, n_last)
        assert np.array_equal(lists[r].cpu().numpy(), want), r


def test_block_selection_without_any_context():
    """Sequences without a context: with and without block selection they attend over their own tokens alone."""
    from paper_2609_33503_b200 import inputs
    from paper_2609_33503_b200.continuations import Continuations
    blk = inputs.BlockShape(hidden=256, inter=384, rope_theta=1.0e4, eps=1.0e-5)
    w = inputs.Workload("continuations", 2, 8, 2, 64, 64, (1,), (1,), 0.15, base_seed=3, planted_chunks=((0,),))
    weights = [inputs.block_weights(w, blk, l, "cuda") for l in range(2)]
    outs = []
    for n_select in (0, 4):
        c = Continuations(8, 2, 64, (0, 0), (1, 2), 2, blk, n_blocks=20, max_len=40, block_size=16, max_rows=24, n_select=n_select)
        c.context_bounds([None] * 2)
        for i, new in enumerate(([20, 1, 3], [1, 1, 0])):
            c.begin(new)
            x = torch.randn(sum(new), 256, generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").to(torch.bfloat16)
            outs.append(c.run(x, weights, [None] * 2).clone())
        assert n_select == 0 or (c.blocks[:2] == -1).all()
    assert status() == B().OK
    for a, b in zip(outs[:2], outs[2:]):
        # two orders of the same bf16 chain: each is some 8e-3 of the exact rows away
        a, b = a.double(), b.double()
        assert torch.isfinite(a).all() and float((a - b).norm() / b.norm()) <= 1.6e-2


def small(seqs=(3,), **kw):
    from paper_2609_33503_b200 import inputs
    from paper_2609_33503_b200.continuations import Continuations
    blk = inputs.BlockShape(hidden=256, inter=384, rope_theta=1.0e4, eps=1.0e-5)
    return Continuations(8, 2, 64, (40,) * len(seqs), seqs, 1, blk, **dict(dict(n_blocks=300, max_len=600, block_size=16, max_rows=40), **kw))


def test_a_step_begins_without_waiting_for_the_steps_before():
    """New counts behind work that takes a quarter of a second: the host goes on at once, and the device's state is the host's copy."""
    c = small()
    c.begin([1, 1, 1])
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    torch.cuda._sleep(500_000_000)
    done.record()
    for new in ([2, 1, 1], [1, 3, 0], [0, 0, 5]):
        c.begin(new)
        assert not done.query()
    torch.cuda.synchronize()
    assert c._len[0].tolist() == c.lens == [4, 5, 7] and c._n_free[0].tolist() == [c.n_free] and status() == B().OK


def test_counts_on_one_stream_are_not_another_streams():
    """Steps on two streams in turn, each behind the other's; what the first stream allocates meanwhile takes no counts' place."""
    c = small()
    side = torch.cuda.Stream()
    main = torch.cuda.current_stream()
    junk = []
    for i in range(150):
        new = [1 + i % 3, (i // 3) % 4, (i // 12) % 5] if i % 10 < 9 else [-1, -1, -1]
        if i % 2:
            side.wait_stream(main)
            with torch.cuda.stream(side):
                torch.cuda._sleep(200_000)
                c.begin(new)
            main.wait_stream(side)
        else:
            c.begin(new)
        if i % 2:
            junk.append(torch.full((3,), 77, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert c._len[0].tolist() == c.lens and c._n_free[0].tolist() == [c.n_free] and status() == B().OK
    assert len(c._new) <= 64


@pytest.mark.parametrize("rows,own", [(3, True), (30, True), (30, False)])
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("mantissa", [1.0, 1.3203125])
@pytest.mark.parametrize("exponent", [10, 21, 33, 60, 104, 124])
def test_the_highest_of_very_large_logits_takes_its_row(rows, own, sign, exponent, mantissa):
    """Logits of some 2^exponent (whose products with the scale are exact in fp32, or are not), one above all others: whatever the number of rows, that key has the weight 1 and its logit is the row's lse.  (The products
    are exact, logits differ by a quarter of their size at least: no rounding can bring another key near.)"""
    b = B()
    D, n = 128, 1500
    for key in (0, 700, n - 1):
        s = Step(8, 2, D, [n], [rows], [17] * rows if own else [0] * rows, 1, 16, seed=22)
        big = 2.0 ** (exponent // 2)
        s.q.zero_()
        s.q[..., 0] = mantissa * 2.0 ** (exponent - exponent // 2)
        k = s.k[s.at[0]:s.at[0] + n]
        k[..., 0] = (sign * big * (1.5 if sign < 0 else 0.5) * (1 + torch.arange(n, device="cuda") % 32 / 128)[:, None]).to(torch.bfloat16)
        k[key, :, 0] = sign * big
        s.ks[..., 0] = sign * big * (1.5 if sign < 0 else 0.5)
        if not own:
            s.row_len = [0] * rows
            s.t["row_len"], s.max_len = i32(s.row_len), 0
        b.relaxkv_shared_prefix_attention(s.shape, s.view, s.store if own else None, s.rows(), s.q, s.out, s.ws(), lse_out=s.lse)
        assert status() == b.OK
        assert torch.equal(s.out.view(rows, 2, 4, D), s.v[s.at[0] + key][None, :, None].expand(rows, 2, 4, D)), key
        want = sign * mantissa * 2.0 ** exponent * float(np.float32(D ** -0.5))
        # fp32: the scale in log2 units, the product, the way back to natural units, twice where pieces are merged; 2^-24 each, with the constants'
        assert float((s.lse.double() / want - 1).abs().max()) <= 8 * 2.0 ** -24, key


def test_steps_in_a_graph_read_counts_that_were_uploaded_before():
    """Two steps as a graph (they use the two sets of lengths in turn); counts that are new to the object are refused while it is captured."""
    c = small()
    for new in ([2, 0, 1], [1, 1, 1]):
        c.begin(new)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.begin([1, 1, 1])
        c.begin([2, 0, 1])
        before = (list(c.lens), c.n_free, c.n_rows, list(c._len))
        with pytest.raises(RuntimeError, match="capture"):
            c.begin([3, 0, 0])
        assert before[:3] == (c.lens, c.n_free, c.n_rows) and all(x is y for x, y in zip(before[3], c._len))
    for i in range(100):                                     # other counts push these out of those that are kept
        c._counts([5 + i, 0, 0])
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert c._len[0].tolist() == c.lens == [6, 2, 4] and c._n_free[0].tolist() == [c.n_free] and status() == B().OK
