"""Chunks of text whose K/V are computed once and used in many contexts: the store that the contexts of a repair are put together from.
(The paper reuses chunks that were prefilled by themselves, Section 2; where they are kept between requests is left to the system around it.)

A chunk lies in 8 bits (half the bytes of the cache it came from) in blocks of one paged store per layer, its keys turned for the positions that they had.
A context takes it back in bf16, its keys turned on to where the chunk begins now, all chunks of it in one launch per layer.

Call sequencing over torch buffers only; every operation runs in the CUDA kernels behind `binding`.
"""
from __future__ import annotations

import dataclasses
from typing import Dict, Hashable, List, Sequence, Tuple

import torch

from . import binding as B


@dataclasses.dataclass(frozen=True)
class _Chunk:
    blocks: Tuple[int, ...]
    slots: torch.Tensor                # int32 [tokens]
    position: int                      # of its first token, as its keys are turned


class ChunkStore:
    """Room for `n_blocks` blocks of `block_size` tokens of all layers.  `rotary` is the embedding of the keys that are kept."""

    def __init__(self, n_layers: int, n_kv_heads: int, head_dim: int, n_blocks: int, rotary: B.Rotary, block_size: int = 64, dtype=torch.int8, device="cuda"):
        self.device, self.block_size = torch.device(device), int(block_size)
        self.stores = [B.QuantizedStore.empty(n_blocks, self.block_size, n_kv_heads, head_dim, dtype, self.device) for _ in range(int(n_layers))]
        # keys that are turned on have their amplitude already
        self.turn = B.Rotary(rotary.freq, rotary.interleaved, 1.0)
        self.free = list(range(int(n_blocks) - 1, -1, -1))
        self.chunks: Dict[Hashable, _Chunk] = {}

    def __contains__(self, key: Hashable) -> bool:
        return key in self.chunks

    def tokens(self, key: Hashable) -> int:
        return int(self.chunks[key].slots.numel())

    def _caches(self, caches: Sequence[B.CacheView], req: int, first: int, n: int) -> None:
        if len(caches) != len(self.stores):
            raise ValueError(f"caches of {len(self.stores)} layers expected, not {len(caches)}")
        for c, s in zip(caches, self.stores):
            if c.v is None or c.heads != s.heads or c.dim != s.dim or not 0 <= req < len(c.room) or first < 0 or first + n > c.tokens(req):
                raise ValueError(f"tokens {first} to {first + n} of request {req} in caches of {s.heads} heads of {s.dim} expected")

    def put(self, key: Hashable, caches: Sequence[B.CacheView], req: int, first: int, n: int, position: int) -> None:
        """Keeps n tokens of a request, from its token `first` on, whose keys are turned for `position` and what follows it."""
        if key in self.chunks:
            raise ValueError(f"there is a chunk {key!r} already")
        if n < 1:
            raise ValueError("a chunk has a token at least")
        self._caches(caches, req, first, n)
        need = -(-n // self.block_size)
        if need > len(self.free):
            raise ValueError(f"{need - len(self.free)} blocks short: let chunks go, or give the store more")
        blocks = self.free[-1:-need - 1:-1]             # (taken when every layer has its rows: a call may be refused)
        slots = torch.tensor([b * self.block_size + t for b in blocks for t in range(self.block_size)][:n], dtype=torch.int32).to(self.device)
        for cache, store in zip(caches, self.stores):
            t = cache.start(req) + first
            B.relaxkv_append_quantized(store, cache.k[t:t + n], cache.v[t:t + n], slots)
        del self.free[-need:]
        self.chunks[key] = _Chunk(tuple(blocks), slots, int(position))

    def drop(self, key: Hashable) -> None:
        """Gives a chunk's blocks back (what has been asked for on the current stream still finds it)."""
        self.free.extend(reversed(self.chunks.pop(key).blocks))

    def assemble(self, keys: Sequence[Hashable], caches: Sequence[B.CacheView], req: int = 0, first: int = 0) -> int:
        """Writes chunks one behind the other into a request's context, from its token `first` on, their keys turned for the positions there (token i of a
        request has position i).  A request reaches to where the next one of the cache begins.  Returns the number of tokens."""
        parts: List[_Chunk] = [self.chunks[k] for k in keys]
        n = sum(int(c.slots.numel()) for c in parts)
        self._caches(caches, req, first, n)
        if n == 0:
            return 0
        at, by = first, []
        for c in parts:
            by.append(at - c.position)
            at += int(c.slots.numel())
        slots = parts[0].slots if len(parts) == 1 else torch.cat([c.slots for c in parts])
        turned = any(by)
        positions = torch.cat([torch.full_like(c.slots, d) for c, d in zip(parts, by)]) if turned else None
        for cache, store in zip(caches, self.stores):
            t = cache.start(req) + first
            B.relaxkv_read_quantized(store, slots, cache.k[t:t + n], cache.v[t:t + n], positions, self.turn if turned else None)
        return n
