"""A paged K/V cache of all layers: the page pools, the page tables and lengths of the sequences in it, and the calls of a serving
loop on them.  Plumbing only: every step is a call of binding.py, in the order of the current stream, and none waits for the GPU.

    cache = PagedCache(n_layers, n_pages, 64, n_kv_heads, head_dim, max_seqs, max_len)
    copies = cache.step(source, add)        # sequences forked, ended, given room for their new rows; pages copied where needed
    for layer in ...:                       # rows of all sequences one after another, row_start[b] the first of sequence b
        q = cache.append(layer, k, v, row_start, q=q, rope_table=table)
        o, lse = cache.attend(layer, q, row_start, scale, max_rows=...)
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as cb


class PagedCache:
    """Pages [n_pages, page_size, n_kv_heads, head_dim] for K and V of every layer, allocated here and nowhere else.  `table`, `kv_len`,
    `refs` and `report` stay the same tensors as long as the cache lives, so a step captured in a graph goes on from one replay to the
    next."""

    def __init__(self, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, max_seqs: int, max_len: int,
                 dtype=torch.bfloat16, device="cuda"):
        self.n_pages, self.page_size = n_pages, page_size
        self.k = [torch.empty((n_pages, page_size, n_kv_heads, head_dim), dtype=dtype, device=device) for _ in range(n_layers)]
        self.v = [torch.empty_like(t) for t in self.k]
        width = -(-max_len // page_size)
        # the table and the lengths in one piece, and a second one for a step to write to
        self._state, self._next = (torch.zeros(max_seqs * (width + 1), dtype=torch.int32, device=device) for _ in range(2))
        (self.table, self.kv_len), (self._next_table, self._next_len) = (
            (t[:max_seqs * width].view(max_seqs, width), t[max_seqs * width:]) for t in (self._state, self._next))
        self.table.fill_(-1)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=device)
        self.report = torch.zeros(4, dtype=torch.int32, device=device)  # of the last step, see cascade_pages_fork

    def step(self, source: torch.Tensor, add: torch.Tensor) -> torch.Tensor:
        """Sequence i goes on as sequence source[i] (int32 on the GPU, -1: none) with room for add[i] more rows, counted in kv_len
        from here on.  Returns the pairs of pages copied.  `report` says whether it could be done; if not, nothing has changed, and
        no rows may be appended."""
        copies = torch.empty((self.kv_len.shape[0], 2), dtype=torch.int32, device=self.table.device)
        cb.cascade_pages_fork(self.table, self.kv_len, source, add, self.n_pages, self.page_size,
                              out=(self._next_table, self._next_len, self.refs, copies, self.report))
        self._copy(copies)
        self._state.copy_(self._next)
        return copies

    def compact(self) -> torch.Tensor:
        """Moves the held pages to the front of the pools; returns (held pages, moves, bad entries, free pages) as int32 [4]."""
        moves = torch.empty((self.n_pages // 2, 2), dtype=torch.int32, device=self.table.device)
        report = torch.empty_like(self.report)
        cb.cascade_pages_compact(self.table, self.kv_len, self.n_pages, self.page_size, out=(self._next_table, self.refs, moves, report))
        self._copy(moves)
        self.table.copy_(self._next_table)
        return report

    def _copy(self, pairs: torch.Tensor) -> None:
        pools = self.k + self.v
        for i in range(0, len(pools), 256):  # as many as a call takes
            cb.cascade_pages_copy(pools[i:i + 256], pairs)

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, row_start: torch.Tensor, q: Optional[torch.Tensor] = None,
               positions=None, rope_table=None, interleaved: bool = False, q_out=None):
        """The new rows of one layer (cascade_paged_append), after step() has made room for them."""
        return cb.cascade_paged_append(k, v, self.k[layer], self.v[layer], self.table, row_start, self.kv_len, q=q,
                                       positions=positions, rope_table=rope_table, interleaved=interleaved, q_out=q_out)

    def attend(self, layer: int, q: torch.Tensor, row_start: torch.Tensor, scale: float, **more):
        """Attention of the new rows of one layer over the cache (cascade_attn_paged): (o, lse)."""
        return cb.cascade_attn_paged(q, self.k[layer], self.v[layer], self.table, row_start, self.kv_len, scale, **more)
