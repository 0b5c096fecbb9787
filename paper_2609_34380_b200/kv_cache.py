"""The key-value cache of a decoder whose blocks a `SumManager` hands out.

The manager decides on the host which KV block of which unit a request gets (and what that does to the residual planes and to
the precision mode); this class keeps what the GPU needs for it: the cache tensors of every layer, one block table for all of
them, and the requests' lengths.  Block (unit, index) of the manager is block id unit * blocks_per_unit + index of the cache.

The requests in hand are rows 0 .. n-1 of a batch.  A step gives each of them new tokens (`extend`: the blocks are taken from the
manager, tables, positions and slots are built by `dps_extend_block_tables`); each layer then writes the step's keys and values
(`write`: `dps_qk_norm_rope` on the QKV linear's output) and, in a step of one token per request, reads all that there are
(`attend`: `dps_paged_attention`).  `finish` gives a request's blocks back and moves the last row into its place.  The tables and
the workspace are one for all calls, which therefore belong on one stream (or streams that events order).
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import binding
from .sum_manager import Block, SumManager


@dataclass
class Step:
    """What one step's kernels read; `single`: every request has one new token, row b of the batch being request b.  Good until the next
    `extend` or `finish`: `lengths` is a view of the cache's own."""
    requests: int
    tokens: int
    single: bool
    lengths: torch.Tensor       # int32 [requests], the new tokens with them
    starts: torch.Tensor        # int32 [requests + 1]
    positions: torch.Tensor     # int32 [rows]
    slots: torch.Tensor         # int64 [rows], -1 behind the last token


class PagedKvCache:
    def __init__(self, manager: SumManager, layers: int, q_heads: int, kv_heads: int, head_dim: int, page_tokens: int, max_requests: int,
                 max_tokens_per_request: int, dtype: torch.dtype = torch.float16) -> None:
        self.manager, self.page_tokens, self.max_requests = manager, page_tokens, max_requests
        self.max_blocks = -(-max_tokens_per_request // page_tokens)
        self.blocks = manager.units * manager.blocks_per_unit
        self.caches = torch.zeros((layers, 2, self.blocks, page_tokens, kv_heads, head_dim), dtype=dtype, device="cuda")
        self.workspace = binding.dps_paged_attention_workspace(q_heads, kv_heads, head_dim)
        self.block_table = torch.full((max_requests, self.max_blocks), -1, dtype=torch.int32, device="cuda")
        self._lengths = torch.zeros((2, max_requests), dtype=torch.int32, device="cuda")   # a step reads one row and writes the other, ...
        self._now = 0                           # ... which is then the one in use
        self._used = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.lengths: List[int] = []            # of the requests in hand, as the host knows them
        self.held: List[List[Block]] = []       # their blocks

    def admit(self) -> int:
        """A new request, without tokens yet; its row."""
        if len(self.lengths) == self.max_requests:
            raise ValueError(f"all {self.max_requests} rows are in use")
        row = len(self.lengths)
        self._lengths[self._now, row] = 0
        self.lengths.append(0)
        self.held.append([])
        return row

    def extend(self, new_tokens: Sequence[int], rows: Optional[int] = None) -> Optional[Step]:
        """Room for new_tokens[b] tokens of each request, or None (and no change) if the manager cannot supply the blocks.  `rows`: the
        step's rows are padded to so many.  A call that raises takes no blocks either."""
        n, total = len(self.lengths), sum(new_tokens)
        if len(new_tokens) != n or any(m < 0 for m in new_tokens):
            raise ValueError(f"one number of new tokens, not negative, for each of the {n} requests")
        rows = total if rows is None else rows
        if rows < total:
            raise ValueError(f"{total} tokens do not fit {rows} rows")
        after = [a + m for a, m in zip(self.lengths, new_tokens)]
        need = [-(-a // self.page_tokens) for a in after]
        if any(b > self.max_blocks for b in need):
            raise ValueError(f"a request would pass {self.max_blocks} blocks")
        fresh = [b - len(h) for b, h in zip(need, self.held)]
        granted = self.manager.alloc_kv_blocks(sum(fresh))
        if granted is None:
            return None
        try:
            ids = [u * self.manager.blocks_per_unit + b for u, b in granted]
            host = torch.tensor([*new_tokens, *ids], dtype=torch.int32).pin_memory()
            both = host.to("cuda", non_blocking=True)
            lengths, starts, positions, slots, _ = binding.dps_extend_block_tables(
                self._lengths[self._now, :n], both[:n], both[n:], self.block_table[:n], self.page_tokens, self.blocks, self._lengths[self._now ^ 1, :n],
                granted_used=self._used, tokens=rows)
        except BaseException:               # no memory for the step, say: nothing was launched, and nobody has the blocks
            self.manager.free_kv_blocks(granted)
            raise
        at = 0
        for held, m in zip(self.held, fresh):
            held.extend(granted[at:at + m])
            at += m
        self._now ^= 1
        self.lengths = after
        return Step(n, total, all(m == 1 for m in new_tokens), lengths, starts, positions, slots)

    def write(self, layer: int, step: Step, qkv: torch.Tensor, cos_sin: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
              k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False) -> torch.Tensor:
        """Keys and values of the step's rows into the layer's cache; the queries, normalised and rotated."""
        k, v = self.caches[layer]
        return binding.dps_qk_norm_rope(qkv, k, v, step.slots, step.positions, cos_sin, q_weight, k_weight, eps, interleaved)

    def attend(self, layer: int, step: Step, q: torch.Tensor, scale: Optional[float] = None) -> torch.Tensor:
        """Attention of each request's one new token over all its tokens; rows behind the requests are left out."""
        if not step.single:
            raise ValueError("attention is for steps of one token per request")
        k, v = self.caches[layer]
        return binding.dps_paged_attention(q[:step.requests], k, v, self.block_table[:step.requests], step.lengths, scale, workspace=self.workspace)

    def finish(self, row: int) -> Optional[int]:
        """The request's blocks go back; the last row takes its place.  Returns that row's former number, None if it was the last itself."""
        last = len(self.lengths) - 1
        if not 0 <= row <= last:
            raise ValueError(f"row {row} is none of the {last + 1} requests")
        self.manager.free_kv_blocks(self.held[row])
        moved = None
        if row != last:
            self.block_table[row] = self.block_table[last]
            self._lengths[self._now, row] = self._lengths[self._now, last]
            self.lengths[row], self.held[row], moved = self.lengths[last], self.held[last], last
        self.lengths.pop()
        self.held.pop()
        return moved
