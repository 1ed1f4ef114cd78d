"""Contexts in 8 bits through the framework's own paths: continuations over them, chunks that contexts are put together from, models with a rotary embedding of their own."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2609_33503_b200 import inputs
from tests import quantized_oracle as orc
from tests.test_gpu_continuations_class import BLK, D, H, HKV, L, rnd, same, setup, status
from tests.test_gpu_quantized import B, TYPES, f64, rotation_tolerance, store_values, value_scale

pytestmark = pytest.mark.gpu


def continuations(*a, **kw):
    from paper_2609_33503_b200.continuations import Continuations

    class Checked(Continuations):
        """Holds every call's attention against the plain form over what the store has then, the appended rows against the formula."""
        checked = 0

        def attention(self, layer, cache, q, out, lse_out=None, stream=None):
            n, store, own = self.n_rows, self.stores[layer], self.block_size
            super().attention(layer, cache, q, out, lse_out, stream)
            kk, vv = store_values(store)
            scales = value_scale(store)
            table, seq, lens, pos, slot = (t.cpu().numpy().astype(np.int64) for t in (self.table, self.row_seq[:n], self.row_len[:n], self.row_pos[:n], self.row_slot[:n]))
            for i in sorted(set(seq)):
                rows = np.flatnonzero(seq == i)
                slots = (table[i, :-(-self.lens[i] // own), None] * own + np.arange(own)).reshape(-1)[:self.lens[i]]
                want, lse, *sizes = orc.attention(f64(q)[rows], kk[slots], vv[slots], lens[rows].tolist(), self.D ** -0.5, scales[slots])
                assert (np.abs(f64(out)[rows] - want) <= orc.attention_tolerance(want, lse, *sizes, self.D)[0]).all()
                assert (pos[rows] == lens[rows] - 1).all() and (slots[pos[rows]] == slot[rows]).all()
            # the appended keys and values: half a step of their exponent (whose step is 2^-6 of the largest element at most), and for keys what fp32 does to them first
            w = self.weights[layer]
            k = orc.turned(f64(self.k[:n]), f64(w["w_k_norm"]), self.blk.eps, pos, self.rotary.freq.cpu().numpy(), self.rotary.interleaved, self.rotary.amplitude)
            for got, want in ((kk[slot], k), (vv[slot], f64(self.v[:n]))):
                step = 2.0 ** -6 if store.k.dtype == torch.int8 else 2.0 ** -3
                assert (np.abs(got - want) <= (step / 2 + 2.0 ** -18) * np.abs(want).max(-1, keepdims=True)).all()
            self.checked += 1

    return Checked(*a, **kw)


@pytest.mark.parametrize("kind", list(TYPES))
def test_questions_and_answers_over_kept_contexts(kind):
    """Two contexts, three sequences: a question each, decoded tokens, an end, the context kept again."""
    ctx = (300, 131)
    weights, caches = setup(ctx, 0)
    c = continuations(H, HKV, D, ctx, (2, 1), L, BLK, n_blocks=60, max_len=40, block_size=16, max_rows=100, store_dtype=TYPES[kind])
    c.weights = weights
    c.keep_contexts(caches)
    assert c.lens == [300, 300, 131] == c._len[0].tolist()
    for i, b in enumerate((0, 0, 1)):                   # what a sequence has is what the cache had, to half a step
        t, n = caches[0].start(b), ctx[b]
        slots = (c.table[i, :-(-n // 16), None] * 16 + torch.arange(16, device="cuda")).reshape(-1)[:n].to(torch.int32)
        for l in range(L):
            k, v = (torch.empty(n, HKV, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            B().relaxkv_read_quantized(c.stores[l], slots, k, v)
            for got, want in ((k, caches[l].k[t:t + n]), (v, caches[l].v[t:t + n])):
                values, e = orc.quantized(f64(want), kind)
                assert (f64(got) == orc.values(values, e)).all()
    for new in ([9, 30, 1], [1, 1, 1], [1, -1, 1]):
        rows = c.begin(new)
        h = c.run(rnd(rows, BLK.hidden, seed=rows), weights)
        assert torch.isfinite(h).all()
    c.keep_contexts(caches, [1])
    c.begin([1, 1, 0])
    c.run(rnd(2, BLK.hidden, seed=9), weights)
    assert c.checked == 4 * L and c.lens == [312, 301, 131 + 3] and status() == B().OK


def test_kept_contexts_in_place_of_caches():
    """Beside the class over bf16 caches.  8 bits move a key or value by up to 2^-7 of its row's largest element (some 3 of its standard deviation), evenly spread: 2^-7 * 3 / sqrt(3) =
    1.4e-2 of its size; a logit (a standard deviation of 1) by 1.4e-2, so a weight by that and what it adds up to by 2e-2; two layers of that on top of two of bf16 arithmetic (1.6e-2)."""
    ctx = (500,)
    weights, caches = setup(ctx, 0)
    from paper_2609_33503_b200.continuations import Continuations
    a = Continuations(H, HKV, D, ctx, (2,), L, BLK, n_blocks=20, max_len=64, block_size=16, max_rows=40)
    b = Continuations(H, HKV, D, ctx, (2,), L, BLK, n_blocks=90, max_len=64, block_size=16, max_rows=40, store_dtype=torch.int8)
    b.keep_contexts(caches)
    for new in ([12, 7], [1, 1]):
        n = a.begin(new)
        assert b.begin(new) == n
        x = rnd(n, BLK.hidden, seed=n)
        want, got = a.run(x, weights, caches).double(), b.run(x, weights).double()
        assert float((got - want).norm() / want.norm()) <= 2 * 2e-2 + 1.6e-2
    assert status() == B().OK


def test_a_captured_step_over_kept_contexts():
    """A step begun and run in a graph, replayed: the sequences grow by a token each time as they do without."""
    ctx = (200,)
    weights, caches = setup(ctx, 0)
    from paper_2609_33503_b200.continuations import Continuations
    make = lambda: Continuations(H, HKV, D, ctx, (2,), L, BLK, n_blocks=40, max_len=64, block_size=16, max_rows=16, store_dtype=torch.float8_e4m3fn)
    plain, graphed = make(), make()
    xs = [rnd(2, BLK.hidden, seed=s) for s in range(4)]
    for c in (plain, graphed):
        c.keep_contexts(caches)
        c.begin([1, 1])
        c.run(xs[0], weights)
    want = []
    plain.begin([1, 1])
    want.append(plain.run(xs[1], weights).clone())
    x = xs[1].clone()
    graphed.begin([1, 1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h = graphed.run(x, weights)
    for _ in range(2):                                  # the same step again: the same rows to the same places
        g.replay()
        assert torch.equal(h, want[0])
    assert status() == B().OK


def test_contexts_put_together_from_chunks():
    """Chunks of two requests, kept where they were computed, put together in another order: keys turned on by how far they moved, values as the store has them."""
    from paper_2609_33503_b200.chunk_store import ChunkStore
    rot = B().Rotary.scaled(64, 5e5, "ramp", 8.0, 4096, 1.0, 32.0, device="cuda")
    weights, caches = setup((300, 200), 0)
    store = ChunkStore(L, HKV, D, 40, rot, block_size=16)
    store.put("a", caches, 0, 0, 100, 0)
    store.put("b", caches, 0, 100, 77, 100)
    store.put("c", caches, 1, 5, 130, 5)
    room = lambda n: [B().CacheView(*(torch.full((n, HKV, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)), [10]) for _ in range(L)]
    keys = ["c", "a", "b", "a"]
    with pytest.raises(ValueError):
        store.assemble(keys, room(400), 0, 3)           # 10 + 3 + 407 tokens
    target = room(430)
    assert store.assemble(keys, target, 0, 3) == 130 + 100 + 77 + 100
    assert rot.amplitude > 1.2
    for l in range(L):
        kk, vv = store_values(store.stores[l])
        at = 13
        for key in keys:
            slots = store.chunks[key].slots.cpu().numpy()
            n = len(slots)
            by = at - 10 - store.chunks[key].position
            k, v = f64(target[l].k[at:at + n]), f64(target[l].v[at:at + n])
            want = orc.turned(kk[slots], None, 0, np.full(n, by), rot.freq.cpu().numpy(), False, 1.0)
            assert (v == vv[slots]).all()
            assert (np.abs(k - want) <= rotation_tolerance(kk[slots], want, None, 1.0)).all()
            at += n
        assert (target[l].k[:13] == 7).all() and (target[l].v[at:] == 7).all()
    store.drop("a")
    store.put("d", caches, 1, 0, 200, 0)                # (its blocks are used again)
    assert store.assemble(["d"], target) == 200         # where it was: as the store has it
    for l in range(L):
        kk, vv = store_values(store.stores[l])
        slots = store.chunks["d"].slots.cpu().numpy()
        assert (f64(target[l].k[10:210]) == kk[slots]).all() and (f64(target[l].v[10:210]) == vv[slots]).all()
        values, e = orc.quantized(f64(caches[l].k[300:500]), "int8")
        assert (kk[slots] == orc.values(values, e)).all()
    assert status() == B().OK


def test_a_rotary_of_the_models_own():
    """The plain embedding as a Rotary gives what rope_theta gives; a scaled one of half a head what the same steps give by themselves (each layer's keys, turned by the formula)."""
    import dataclasses

    from paper_2609_33503_b200.continuations import Continuations
    from paper_2609_33503_b200.query_pass import QueryPass
    ctx, qn = (150, 70), (9, 4)
    results = []
    plain = B().Rotary.scaled(D, BLK.rope_theta)
    half = B().Rotary.scaled(D // 2, BLK.rope_theta, "bands", 8.0, 128, 1.0, 4.0, interleaved=True)
    for rotary in (None, plain, half):
        blk = dataclasses.replace(BLK, rotary=rotary)
        weights, caches = setup(ctx, 16)
        qp = QueryPass(H, HKV, D, ctx, qn, blk, extra_tokens=4)
        c = Continuations(H, HKV, D, ctx, (1, 1), L, blk, n_blocks=6, max_len=40, block_size=16, max_rows=16)
        x = rnd(sum(qn), BLK.hidden, seed=1)
        h = qp.prefill(x, weights, caches).clone()
        c.begin(qn)
        assert same(c.run(x, weights, caches), h)
        results.append(h)
        if rotary is not None:                          # the last layer's queries as the pass has left them: norm and rotation are in the keys that lie in cache and store
            n, pos = sum(qn), np.concatenate([np.arange(t, t + q) for t, q in zip(ctx, qn)])
            slot = c.row_slot[:n].cpu().numpy()
            hh, w = rnd(sum(qn), BLK.hidden, seed=1), weights[0]
            normed, q, k, v = torch.empty_like(hh), torch.empty(n, H, D, **bf16()), torch.empty(n, HKV, D, **bf16()), torch.empty(n, HKV, D, **bf16())
            B().relaxkv_rmsnorm(hh, w["w_in_norm"], normed, blk.eps)
            B().relaxkv_linear_qkv(normed, w["w_qkv"], q, k, v)
            want = orc.turned(f64(k), f64(w["w_k_norm"]), blk.eps, pos, rotary.freq.cpu().numpy(), rotary.interleaved, rotary.amplitude)
            tol = rotation_tolerance(f64(k), want, w["w_k_norm"], rotary.amplitude)
            cached = torch.cat([caches[0].k[caches[0].start(b) + t:caches[0].start(b) + t + q_] for b, (t, q_) in enumerate(zip(ctx, qn))])
            stored = c.stores[0].k.reshape(-1, HKV, D)[torch.tensor(slot, device="cuda").long()]
            assert (np.abs(f64(cached) - want) <= tol).all() and (np.abs(f64(stored) - want) <= tol).all()
    assert same(results[1], results[0]) and not same(results[2], results[0])
    assert status() == B().OK


def bf16():
    return dict(dtype=torch.bfloat16, device="cuda")


def test_a_repair_with_a_rotary_of_the_models_own():
    """The repair loop of a model whose embedding is given as a Rotary: as with the same embedding by its theta."""
    import dataclasses

    from paper_2609_33503_b200.layer_loop import LayerLoop
    from paper_2609_33503_b200.pipeline import RepairSession
    w = inputs.Workload("repair", L, H, HKV, D, 64, (512,), (16,), 0.15, base_seed=3, planted_chunks=((1,),))
    out = []
    for rotary in (None, B().Rotary.scaled(D, BLK.rope_theta)):
        blk = dataclasses.replace(BLK, rotary=rotary)
        weights = [inputs.block_weights(w, blk, l, "cuda") for l in range(L)]
        layers = [inputs.layer_qkv(w, l, 0, "cuda") for l in range(L)]
        caches = [B().CacheView(k, v, [0]) for _, k, v in layers]
        s = RepairSession(H, HKV, D, [512], [16], L, [B().relaxkv_anchor_count(512, 0.15)])
        s.score_select([q for q, _, _ in layers], caches)
        s.build_active_sets()
        n_u, _ = s.counts()
        h0 = inputs.input_representations(w, blk, 0, s.u_pos[:n_u[0]], "cuda")
        out.append((LayerLoop(s, blk, s.cap_u).run(h0, weights, caches).clone(), caches[0].k.clone()))
    assert same(out[1][0], out[0][0]) and same(out[1][1], out[0][1]) and status() == B().OK


def test_the_example_runs_over_kept_contexts():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for store in ("int8", "e4m3"):
        r = subprocess.run([sys.executable, os.path.join(root, "examples", "sample_answers.py"), "--ctx", "2048", "--layers", "2", "--samples", "3", "--steps", "3", "--store", store],
                           capture_output=True, text=True, timeout=300, cwd=root)
        assert r.returncode == 0, r.stderr[-2000:]
        assert "3 samples of a context of 2048 tokens" in r.stdout
