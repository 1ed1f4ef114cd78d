"""Steps over contexts that are kept in 8 bits, begun and run in a captured graph."""
import pytest
import torch

from tests.test_gpu_continuations_class import BLK, D, H, HKV, L, rnd, setup, status
from tests.test_gpu_quantized import B, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(TYPES))
def test_steps_begun_in_a_graph_go_on(kind):
    """Two steps as a graph (they use the two sets of lengths in turn): each replay appends two tokens to every sequence, as steps without a graph do."""
    from paper_2609_33503_b200.continuations import Continuations
    ctx = (200, 33)
    weights, caches = setup(ctx, 0)
    make = lambda: Continuations(H, HKV, D, ctx, (2, 1), L, BLK, n_blocks=60, max_len=64, block_size=16, max_rows=16, store_dtype=TYPES[kind])
    plain, graphed = make(), make()
    xs = [rnd(3, BLK.hidden, seed=s) for s in range(2)]
    for c in (plain, graphed):
        c.keep_contexts(caches)
        c.begin([1, 1, 1])
        c.run(xs[0], weights)
    graphed.begin([1, 1, 1])
    graphed.run(xs[1], weights)
    plain.begin([1, 1, 1])
    plain.run(xs[1], weights)
    torch.cuda.synchronize()
    graph, outs = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        for x in xs:
            graphed.begin([1, 1, 1])
            outs.append(graphed.run(x, weights).clone())
    graph.replay()
    want = []
    for x in xs:
        plain.begin([1, 1, 1])
        want.append(plain.run(x, weights).clone())
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert graphed._len[0].tolist() == plain._len[0].tolist() == [204, 204, 37] == graphed.lens and status() == B().OK
