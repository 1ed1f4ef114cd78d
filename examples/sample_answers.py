"""Several answers from one repaired context: a request's context is repaired (scores, anchors, sparse-context attention, cache update), then
`--samples` continuations of it are decoded side by side.  Synthetic states and weights; prints the time of each part.

    python examples/sample_answers.py                       # 16 samples of a 16K context, 4 layers of 32 / 8 heads
    python examples/sample_answers.py --select 64           # each row reads the 64 context blocks it may need most
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_33503_b200 import binding as B  # noqa: E402
from paper_2609_33503_b200 import inputs  # noqa: E402
from paper_2609_33503_b200.continuations import Continuations  # noqa: E402
from paper_2609_33503_b200.layer_loop import LayerLoop  # noqa: E402
from paper_2609_33503_b200.pipeline import RepairSession  # noqa: E402


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--ctx", type=int, default=16384)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--samples", type=int, default=16)
    ap.add_argument("--steps", type=int, default=16, help="decoded tokens per sample")
    ap.add_argument("--question", type=int, default=8, help="tokens of the question that every sample begins with")
    ap.add_argument("--select", type=int, default=0, help="context blocks that a row reads (0: the whole context)")
    a = ap.parse_args()
    H, Hkv, D, L, ctx = 32, 8, 128, a.layers, a.ctx
    blk = inputs.BlockShape(hidden=1024, inter=2048, rope_theta=5.0e5, eps=1.0e-5)
    w = inputs.Workload("answers", L, H, Hkv, D, 512, (ctx,), (a.question,), 0.15, base_seed=1, planted_chunks=((0,),))
    weights = [inputs.block_weights(w, blk, l, "cuda") for l in range(L)]
    q_layers, caches = [], []
    for l in range(L):
        q, k, v = inputs.layer_qkv(w, l, 0, "cuda")
        q_layers.append(q)
        caches.append(B.CacheView(k, v, [0]))
    timed = []

    def span(name, fn):
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        out = fn()
        t1.record()
        timed.append((name, t0, t1))
        return out

    # ---- the repair: scores and anchors, schedule, the loop over the layers with the cache update ----
    s = RepairSession(H, Hkv, D, [ctx], [a.question], L, [B.relaxkv_anchor_count(ctx, 0.15)])

    def repair():
        s.score_select(q_layers, caches)
        s.build_active_sets()
        n_u, _ = s.counts()
        h0 = inputs.input_representations(w, blk, 0, s.u_pos[:n_u[0]], "cuda")
        LayerLoop(s, blk, s.cap_u).run(h0, weights, caches)

    span("repair", repair)

    # ---- the samples: the question once each, then one token of each per step ----
    n = a.samples
    c = Continuations(H, Hkv, D, [ctx], [n], L, blk, n_blocks=n * (-(-(a.question + a.steps) // 16)), max_len=a.question + a.steps, block_size=16,
                      max_rows=n * max(1, a.question), n_select=a.select)
    span("bounds", lambda: c.context_bounds(caches))
    g = torch.Generator(device="cuda").manual_seed(7)
    embed = lambda rows: torch.randn(rows, blk.hidden, generator=g, device="cuda").to(torch.bfloat16)
    question = embed(a.question).repeat(n, 1)

    def ask():
        c.begin([a.question] * n)
        return c.run(question, weights, caches)

    h = span("question", ask).view(n, a.question, -1)
    # (equal rows in other places of a tile are not always summed in the same order)
    spread = float((h.float() - h[:1].float()).abs().max())

    def step():
        c.begin([1] * n)
        return c.run(embed(n), weights, caches)

    for i in range(a.steps):
        h = span(f"step {i}", step)
    torch.cuda.synchronize()
    status = B.relaxkv_read_device_status()[0]
    assert status == B.OK, B.status_string(status)
    assert torch.isfinite(h.float()).all() and spread < 0.25, spread
    ms = {name: t0.elapsed_time(t1) for name, t0, t1 in timed}
    print(f"{n} samples of a context of {ctx} tokens, {L} layers: repair {ms['repair']:.2f} ms, question {ms['question']:.2f} ms, last step "
          f"{ms[f'step {a.steps - 1}']:.3f} ms, {c.n_free} blocks left")


if __name__ == "__main__":
    main()
