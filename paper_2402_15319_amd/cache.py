"""The pages of a decoder's key-value cache and who holds them: host bookkeeping around vq_cache_copy.

Sequences take pages from one pool as they grow, share them after a fork, give them back when they are freed.  A page that
several sequences share is copied when one of them writes into it; compaction moves the pages in use to the lowest numbers.
Buffers, copies and the batches for the attention calls go by the same page numbers in every layer.

Copies are enqueued on the stream given (by default the current one of the cache's GPU): use the cache on one stream, or order the streams.
"""
from __future__ import annotations

import contextlib
import heapq

import torch

from . import VQ_BF16, VQ_F16, AttnBatch, make_attn_desc, vq_cache_copy

__all__ = ["PagedCache", "OutOfPages"]


class OutOfPages(RuntimeError):
    """The pool has fewer free pages than asked for; nothing has changed."""


class PagedCache:
    """layers: how many K and V buffers there are; table_width: pages a sequence may have (its length is at most
    table_width * page_size).  k[layer] and v[layer] are the buffers, desc the descriptor for the attention calls."""

    def __init__(self, layers: int, heads: int, kv_heads: int, head_dim: int, page_size: int, n_pages: int, table_width: int,
                 dtype: int = VQ_F16, scale: float | None = None, device="cuda:0"):
        if layers < 1 or n_pages < 1 or table_width < 1:
            raise ValueError("PagedCache: layers, n_pages and table_width are positive")
        if dtype not in (VQ_F16, VQ_BF16):
            raise ValueError("PagedCache: dtype is VQ_F16 or VQ_BF16")
        self.desc = make_attn_desc(heads, kv_heads, head_dim, page_size, n_pages, dtype, scale)
        self.page_size, self.n_pages, self.table_width, self.device = page_size, n_pages, table_width, device
        kind = torch.float16 if dtype == VQ_F16 else torch.bfloat16
        self.k = [torch.empty(n_pages, kv_heads, page_size, head_dim, dtype=kind, device=device) for _ in range(layers)]
        self.v = [torch.empty(n_pages, kv_heads, head_dim, page_size, dtype=kind, device=device) for _ in range(layers)]
        self._buffers = self.k + self.v
        self._free = list(range(n_pages))   # a heap: the lowest numbers are given out first
        self._holders = [0] * n_pages       # sequences that list a page
        self._pages: dict[int, list[int]] = {}
        self._length: dict[int, int] = {}
        self._next = 0

    # ------------------------------------------------------------------ sequences
    def add(self) -> int:
        """A new, empty sequence; its number."""
        s = self._next
        self._next += 1
        self._pages[s], self._length[s] = [], 0
        return s

    def length(self, s: int) -> int:
        return self._length[s]

    def pages(self, s: int) -> list[int]:
        return list(self._pages[s])

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def fork(self, s: int) -> int:
        """A new sequence with the tokens of s, in the same pages."""
        pages, length = list(self._pages[s]), self._length[s]
        t = self.add()
        self._pages[t], self._length[t] = pages, length
        for p in self._pages[t]:
            self._holders[p] += 1
        return t

    def free(self, s: int) -> None:
        """Forgets s; pages that nobody else holds go back to the pool."""
        for p in self._pages.pop(s):
            self._holders[p] -= 1
            if self._holders[p] == 0:
                heapq.heappush(self._free, p)
        del self._length[s]

    def grow(self, sequences, new, stream=None) -> None:
        """Room for new[i] more tokens in sequences[i] (each named once); their lengths count them from here on.  A last page
        that is shared and not full is copied first: one vq_cache_copy for all of them."""
        sequences, new = list(sequences), list(new)
        if len(sequences) != len(new) or len(set(sequences)) != len(sequences) or any(n < 0 for n in new):
            raise ValueError("grow: as many counts (not negative) as sequences, each sequence once")
        shared: dict[int, int] = {}         # holders that a shared last page loses to copies made here
        plan, want = [], 0
        for s, n in zip(sequences, new):
            have = len(self._pages[s])
            need = -(-(self._length[s] + n) // self.page_size)
            if need > self.table_width:
                raise ValueError(f"grow: sequence {s} would need {need} pages, its table has {self.table_width}")
            copy = False
            if n and self._length[s] % self.page_size:
                last = self._pages[s][-1]
                copy = self._holders[last] - shared.get(last, 0) > 1
                shared[last] = shared.get(last, 0) + copy
            plan.append((s, n, copy, need - have))
            want += copy + need - have
        if want > len(self._free):
            raise OutOfPages(f"{want} pages wanted, {len(self._free)} free")
        taken = [heapq.heappop(self._free) for _ in range(want)]
        ahead = iter(taken)
        chosen = [(next(ahead) if copy else None, [next(ahead) for _ in range(more)]) for _, _, copy, more in plan]
        pairs = [(self._pages[s][-1], page) for (s, _, _, _), (page, _) in zip(plan, chosen) if page is not None]
        if pairs:
            try:
                self._copy(pairs, stream)
            except BaseException:
                for page in taken:
                    heapq.heappush(self._free, page)
                raise
        for (s, n, _, _), (page, more) in zip(plan, chosen):
            own = self._pages[s]
            if page is not None:
                self._holders[own[-1]] -= 1
                own[-1] = page
            own.extend(more)
            self._length[s] += n
        for page in taken:
            self._holders[page] = 1

    def compact(self, stream=None) -> int:
        """Moves the pages in use to the lowest numbers; how many moved.  Batches made before list the old numbers."""
        used = self.n_pages - len(self._free)
        holes = sorted(p for p in self._free if p < used)
        moved = [p for p in range(used, self.n_pages) if self._holders[p]]
        pairs = list(zip(moved, holes))
        if pairs:
            self._copy(pairs, stream)
            to = dict(pairs)
            for own in self._pages.values():
                own[:] = [to.get(p, p) for p in own]
            for a, b in pairs:
                self._holders[b], self._holders[a] = self._holders[a], 0
        self._free = list(range(used, self.n_pages))   # sorted, so a heap
        return len(pairs)

    def _copy(self, pairs, stream) -> None:
        device = torch.device(self.device)
        with torch.cuda.device(device) if device.type == "cuda" else contextlib.nullcontext():
            vq_cache_copy(self.desc, self._buffers, pairs, stream=stream)

    # ------------------------------------------------------------------ calls
    def batch(self, sequences, new=None) -> AttnBatch:
        """The AttnBatch of these sequences with new[i] new tokens each, which their lengths already count (None: one each)."""
        sequences = list(sequences)
        lens = [self._length[s] for s in sequences]
        width = max([1] + [len(self._pages[s]) for s in sequences])
        table = [self._pages[s] + [-1] * (width - len(self._pages[s])) for s in sequences]
        put = lambda x: torch.tensor(x, dtype=torch.int32).to(self.device)  # noqa: E731
        if new is None:
            return AttnBatch(put(lens), put(table), max_len=max(lens))
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        return AttnBatch(put(lens), put(table), n_tokens=starts[-1], max_len=max(lens), q_start=put(starts))
