"""Many continuations of repaired contexts: several samples or follow-up questions that share what a repair has paid for.
(The paper answers one query per repair; this is its decode step for callers that answer from one repaired context many times.)

The contexts stay in the caches the repair loop leaves them in.  What a continuation ("sequence") adds of its own - a question, the
answer so far - lives in blocks of a paged store, one per layer, handed out on the GPU.  A step appends some tokens to some sequences: block
tables and slot maps once for all layers, then per layer the decoder block, with norm, rotation and append of the rows' K/V in one
launch and attention over [the shared context, the sequence's own tokens].  The context is read once for all its rows; with
`n_select` only the blocks that each row may need most are read (8-bit bounds of the keys' blocks choose them).

Call sequencing over torch buffers only; every operation runs in the CUDA kernels behind `binding`.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Sequence

import torch

from . import binding as B
from .inputs import BlockShape


class Continuations:
    """Sequences over the contexts of a batch: `seqs[b]` of them continue context b (`ctx_lens[b]` tokens; 0: none).  Room for
    `n_blocks` blocks of `block_size` own tokens in all, `max_len` to a sequence, and steps of up to `max_rows` rows."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, ctx_lens: Sequence[int], seqs: Sequence[int], n_layers: int,
                 blk: BlockShape, n_blocks: int, max_len: int, block_size: int = 64, max_rows: Optional[int] = None, n_select: int = 0,
                 n_first: int = 1, n_last: int = 2, ctx_block: int = 64, device="cuda", softmax_scale: Optional[float] = None):
        self.H, self.Hkv, self.D, self.blk, self.n_layers = n_q_heads, n_kv_heads, head_dim, blk, int(n_layers)
        self.device = torch.device(device)
        self.ctx_lens, self.seqs = [int(x) for x in ctx_lens], [int(x) for x in seqs]
        self.seq_cu = [sum(self.seqs[:b]) for b in range(len(self.seqs) + 1)]
        n_seq = self.n_seq = self.seq_cu[-1]
        self.max_rows = n_seq if max_rows is None else int(max_rows)
        self.block_size, self.ctx_block = int(block_size), int(ctx_block)
        self.n_select, self.n_first, self.n_last = int(n_select), int(n_first), int(n_last)
        self.shape = B.Shape(self.H, self.Hkv, self.D, self.ctx_lens, None, softmax_scale)
        bf = dict(dtype=torch.bfloat16, device=self.device)
        i32 = dict(dtype=torch.int32, device=self.device)
        self.stores = [B.PagedStore(*(torch.empty(n_blocks, self.block_size, self.Hkv, self.D, **bf) for _ in range(2)))
                       for _ in range(self.n_layers)]
        self.width = -(-int(max_len) // self.block_size)
        self.table = torch.full((n_seq, self.width), -1, **i32)
        self.free = torch.arange(n_blocks - 1, -1, -1, **i32)
        self._n_free = [torch.full((1,), n_blocks, **i32), torch.empty(1, **i32)]          # before and after a step, in turn
        self._len = [torch.zeros(n_seq, **i32), torch.empty(n_seq, **i32)]
        self.base = torch.cat([torch.full((n,), t, **i32) for t, n in zip(self.ctx_lens, self.seqs)] or [torch.empty(0, **i32)])
        self.lens = [0] * n_seq                        # the host's copy of the lengths: what it asks for is what it gets
        self.n_free = int(n_blocks)
        self._new: Dict[tuple, torch.Tensor] = {}
        self._captured: List[torch.Tensor] = []
        R = self.max_rows
        self.row_cu = torch.empty(n_seq + 1, **i32)
        self.row_seq, self.row_pos, self.row_len, self.row_slot = (torch.empty(R, **i32) for _ in range(4))
        e = lambda *s: torch.empty(*s, **bf)
        C, I = blk.hidden, blk.inter
        self.x, self.a, self.h = e(R, C), e(R, C), [e(R, C), e(R, C)]
        self.q, self.k, self.v, self.o = e(R, self.H, self.D), e(R, self.Hkv, self.D), e(R, self.Hkv, self.D), e(R, self.H, self.D)
        self.gu, self.m = e(R, 2 * I), e(R, I)
        self.bounds = self.scale = self.blocks = None
        if self.n_select > 0:
            nb = sum(-(-t // self.ctx_block) for t in self.ctx_lens)
            self.bounds = [torch.empty(nb, self.Hkv, 2, self.D, dtype=torch.int8, device=self.device) for _ in range(self.n_layers)]
            self.scale = [torch.empty(nb, self.Hkv, dtype=torch.float32, device=self.device) for _ in range(self.n_layers)]
            self.blocks = torch.empty(R, self.Hkv, self.n_select, **i32)
        nbytes = B.relaxkv_continuation_workspace_bytes(self.shape, R, self.ctx_block if self.n_select else 0)
        if nbytes == 0:
            raise B.RelaxKVError(B.ERR_INVALID_ARG, "relaxkv_continuation_workspace_bytes")
        ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        off = (-ws.data_ptr()) % 256
        self.workspace = ws[off:off + nbytes]
        self.rows: Optional[B.ContinuationRows] = None
        self.n_rows = 0

    def context_bounds(self, caches: Sequence[B.CacheView], stream=None) -> None:
        """Bounds of the context blocks of every layer, for `n_select`: once, when the repair has left the caches as they are to be read."""
        for l in range(self.n_layers if self.n_select else 0):
            B.relaxkv_block_bounds(self.shape, caches[l], self.ctx_block, self.bounds[l], self.scale[l], stream=stream)

    def _rows(self, h: torch.Tensor, n: int) -> torch.Tensor:
        """The first n hidden rows of h: the kernels take as many as the buffers beside them have."""
        if h.dim() != 2 or h.shape[0] < n or h.shape[1] != self.blk.hidden or h.dtype != torch.bfloat16 or not h.is_contiguous():
            raise ValueError(f"{n} contiguous bf16 rows of {self.blk.hidden} expected, not {tuple(h.shape)} of {h.dtype}")
        return h if h.shape[0] == n else h[:n]

    def _blocks(self, tokens: int) -> int:
        return -(-tokens // self.block_size)

    def _counts(self, new: List[int]) -> torch.Tensor:
        """The counts on the device, by way of pinned memory: the host waits for nothing.  Those of the last steps are kept for the stream that
        they were uploaded on (a stream's memory is handed out again in its own order)."""
        key = (B._stream(None), *new)
        if self.device.type == "cuda" and torch.cuda.is_current_stream_capturing():
            # a graph reads what an earlier step has uploaded, as long as this object lives: its own copy would read pinned memory that is used again
            known = next((t for k, t in self._new.items() if k[1:] == key[1:]), None)
            if known is None:
                raise RuntimeError("a step whose counts are new cannot begin in a graph's capture: begin one of the same counts before")
            self._captured.append(known)
            return known
        if key not in self._new:
            if len(self._new) >= 64:
                del self._new[next(iter(self._new))]
            host = torch.tensor(new, dtype=torch.int32, pin_memory=self.device.type == "cuda")
            self._new[key] = host.to(self.device, non_blocking=True)
        return self._new[key]

    def begin(self, new: Sequence[int]) -> int:
        """Begins a step: new[i] tokens of sequence i follow (0: it waits, -1: it ends and gives its blocks back).  Block tables, positions and
        slots of the rows are made on the device, on the current stream; the rows are those of the sequences in order.  Returns their number."""
        new = [int(x) for x in new]
        if len(new) != self.n_seq or any(n < -1 for n in new):
            raise ValueError(f"a step of {self.n_seq} sequences takes as many counts, -1 or more each")
        lens = [0 if n < 0 else t + n for t, n in zip(self.lens, new)]
        rows = sum(n for n in new if n > 0)
        # what the device would refuse is refused here, before anything has changed
        if rows > self.max_rows:
            raise ValueError(f"{rows} rows in a step of at most {self.max_rows}")
        if any(t > self.width * self.block_size for t in lens):
            raise ValueError(f"a sequence of {max(lens)} tokens with room for {self.width * self.block_size}")
        n_free = self.n_free + sum(self._blocks(t) for t in self.lens) - sum(self._blocks(t) for t in lens)
        if n_free < 0:
            raise ValueError(f"{-n_free} blocks short: let sequences end, or give the store more")
        B.relaxkv_build_block_tables(self.block_size, self._len[0], self._counts(new), self.base, self.free, self._n_free[0], self.table,
                                     self._len[1], self._n_free[1], self.row_cu, self.row_seq[:rows], self.row_pos[:rows],
                                     self.row_len[:rows], self.row_slot[:rows])
        self._len.reverse()
        self._n_free.reverse()
        self.lens, self.n_free, self.n_rows = lens, n_free, rows
        per_ctx = [sum(n for n in new[a:b] if n > 0) for a, b in zip(self.seq_cu, self.seq_cu[1:])]
        longest = max([t for t, n in zip(lens, new) if n > 0], default=0)
        self.rows = B.ContinuationRows(self.seq_cu, per_ctx, longest, self.row_cu, self.row_seq[:rows], self.row_len[:rows], self.table)
        return rows

    def attention(self, layer: int, cache: Optional[B.CacheView], q: torch.Tensor, out: torch.Tensor, lse_out=None, stream=None) -> None:
        """Attention of the step's rows at one layer, their own K/V appended: over the whole contexts, or over n_select blocks of them."""
        if self.n_select == 0:
            B.relaxkv_shared_prefix_attention(self.shape, cache, self.stores[layer], self.rows, q, out, self.workspace, lse_out=lse_out, stream=stream)
            return
        blocks = self.blocks[:self.n_rows]
        B.relaxkv_select_blocks(self.shape, self.ctx_block, self.bounds[layer], self.scale[layer], self.rows, q, self.n_first, self.n_last, blocks,
                                self.workspace, stream=stream)
        B.relaxkv_block_sparse_attention(self.shape, cache, self.stores[layer], self.rows, self.ctx_block, blocks, q, out, self.workspace,
                                         lse_out=lse_out, stream=stream)

    def run(self, h0: torch.Tensor, weights: List[Dict[str, torch.Tensor]], caches: Sequence[Optional[B.CacheView]]) -> torch.Tensor:
        """The step's rows through the decoder: h0 [n_rows, hidden] = their input representations (rows behind them are not looked
        at).  Returns the hidden rows after the last layer (one of this object's buffers)."""
        n, blk = self.n_rows, self.blk
        if n == 0:
            return h0
        x, a, q, k, v, o, gu, m = (t[:n] for t in (self.x, self.a, self.q, self.k, self.v, self.o, self.gu, self.m))
        h = self._rows(h0, n)
        for l, w in enumerate(weights):
            if "w_qkv" not in w:                        # weight-loading steps, once per layer
                w["w_qkv"] = B.stack_qkv(w["wq"], w["wk"], w["wv"])
            if blk.inter % 128 == 0 and "w_gate_up_tiled" not in w:
                w["w_gate_up_tiled"] = B.tile_gate_up(w["w_gate_up"])
            h_out = self.h[l % 2][:n]
            B.relaxkv_rmsnorm(h, w["w_in_norm"], x, blk.eps)
            B.relaxkv_linear_qkv(x, w["w_qkv"], q, k, v)
            B.relaxkv_qk_norm_rope_append_paged(self.stores[l], q, k, v, self.row_pos, self.row_slot, blk.rope_theta, q, w.get("w_q_norm"),
                                                w.get("w_k_norm"), blk.eps)
            self.attention(l, caches[l], q, o)
            B.relaxkv_linear(o, w["wo"], a, residual=h)
            B.relaxkv_rmsnorm(a, w["w_post_norm"], x, blk.eps)
            if blk.inter % 128 == 0:
                B.relaxkv_linear_swiglu(x, w["w_gate_up_tiled"], m)
            else:
                B.relaxkv_linear(x, w["w_gate_up"], gu)
                B.relaxkv_swiglu(gu, m)
            B.relaxkv_linear(m, w["w_down"], h_out, residual=a)
            h = h_out
        return h

    def output_head(self, h: torch.Tensor, final_norm: torch.Tensor, w_head: torch.Tensor, logits: torch.Tensor) -> torch.Tensor:
        """Final RMSNorm and output projection of the given rows: logits [rows, vocab]."""
        n, vocab = h.shape[0], w_head.shape[0]
        if n > self.max_rows or w_head.shape[1] != self.blk.hidden:
            raise ValueError(f"{n} rows of at most {self.max_rows} by a head {tuple(w_head.shape)}")
        if logits.numel() < n * vocab or logits.dtype != torch.bfloat16 or not logits.is_contiguous():
            raise ValueError(f"logits of {n} contiguous bf16 rows of {vocab} expected, not {tuple(logits.shape)} of {logits.dtype}")
        h, x = self._rows(h, n), self.x[:n]
        B.relaxkv_rmsnorm(h, final_norm, x, self.blk.eps)
        B.relaxkv_linear(x, w_head, logits)
        return logits
