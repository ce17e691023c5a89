"""A sequence cache in pages of 8 bits for serving: half the bytes of a decode step over bf16 pages, and with selected blocks a small part of them.

The mechanisms are the library's: ``moda_kv_write_e4m3`` quantises new rows into the pages, ``moda_kv_read_e4m3`` gives them back for the prefill of a later chunk,
``moda_kv_select_blocks`` picks the blocks of 64 positions that a token attends to, ``moda_attn_decode_e4m3`` is the step over all or the picked blocks.  This class
keeps the pages, which sequence has which, and the lengths.

    cache = PagedCache(B, H_kv, d, num_pages=4096, max_len=131072)
    cache.write(K, V)                                    # a prompt's rows [B, T, H_kv, d], or n_new[b] <= T of each
    for token in ...:
        cache.write(k[:, None], v[:, None])              # the token's own key and value
        O, LSE = cache.attend(q, depth_kv_token, l, scale)                               # every position
        O, LSE = cache.attend(q, depth_kv_token, l, scale, n_blocks=64, n_recent=2)      # 64 blocks of every (sequence, key/value head)
    cache.release(b)                                     # sequence b has ended: its pages are free, its place is empty

The host decides which page a sequence gets, so it knows every length: ``n_new`` is a list of numbers.  Positional information has to be in the keys.
``attend`` and ``select`` can be captured into a CUDA graph: a replay takes the lengths and pages of its time, up to ``longest`` positions.  ``write`` and ``release`` cannot.
"""
from __future__ import annotations

import torch

from . import binding


class PagedCache:
    def __init__(self, B: int, H_kv: int, d: int, num_pages: int, max_len: int, page_size: int = 64, bounds: bool = True, device="cuda"):
        if B < 1 or max_len < 1:
            raise ValueError("B >= 1 and max_len >= 1 required")
        self.B, self.H_kv, self.d, self.page_size, self.max_len = B, H_kv, d, page_size, max_len
        self.pages = binding.alloc_kv_pages_e4m3(num_pages, page_size, H_kv, d, device)
        self.bounds = binding.alloc_kv_bounds(num_pages, page_size, H_kv, d, device) if bounds else None
        self.most = -(-max_len // page_size)                   # pages of a sequence
        self.table = torch.full((B, self.most), -1, device=device, dtype=torch.int32)
        self.lens = torch.zeros((B,), device=device, dtype=torch.int32)
        self.lengths = [0] * B                                 # what `lens` holds
        self._owned = [[] for _ in range(B)]
        self._free = list(range(num_pages - 1, -1, -1))
        self._turns = [0] * B                                  # sequences that have had each place before
        self.index = None                                      # of the last selection

    @property
    def longest(self) -> int:
        return max(self.lengths)

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def _reserve(self, n_new):
        """Pages for n_new[b] more positions of every sequence, as a list a sequence, or an error.  They are still free: ``_take`` them."""
        need = []
        for b, n in enumerate(n_new):
            end = self.lengths[b] + n
            if end > self.max_len:
                raise ValueError(f"sequence {b} would have {end} positions, the cache is for {self.max_len}")
            need.append(max(-(-end // self.page_size) - len(self._owned[b]), 0))
        if sum(need) > len(self._free):
            raise ValueError(f"{sum(need)} pages required, {len(self._free)} are free")
        free = iter(reversed(self._free))
        return [[next(free) for _ in range(n)] for n in need]

    def _enter(self, pages, taken=True):
        """Into the table, behind those of each sequence (or out of it again)."""
        at = [b * self.most + len(self._owned[b]) + i for b, own in enumerate(pages) for i in range(len(own))]
        if at:
            device, number = self.table.device, [p if taken else -1 for own in pages for p in own]
            self.table.view(-1).index_copy_(0, torch.tensor(at, device=device), torch.tensor(number, device=device, dtype=torch.int32))

    def _take(self, pages):
        for own, more in zip(self._owned, pages):
            own.extend(more)
            del self._free[len(self._free) - len(more):]

    def write(self, K, V, n_new=None):
        """Appends the first ``n_new[b]`` (None: all T) rows of K, V [B,T,H_kv,d] to every sequence."""
        if K.dim() != 4 or (K.shape[0], K.shape[2], K.shape[3]) != (self.B, self.H_kv, self.d):
            raise ValueError("K must be [B, T, H_kv, d] of this cache")
        T = K.shape[1]
        count = [T] * self.B if n_new is None else [int(n) for n in n_new]
        if len(count) != self.B or min(count) < 0 or max(count) > T:
            raise ValueError("n_new must be B numbers from 0 to T")
        if K.shape != V.shape or K.dtype != torch.bfloat16 or V.dtype != torch.bfloat16 or not (K.is_contiguous() and V.is_contiguous()):
            raise ValueError("K and V must be contiguous bf16 tensors of one shape")
        if max(count) == 0:
            return
        pages = self._reserve(count)
        self._enter(pages)
        try:
            more = None if n_new is None else torch.tensor(count, device=self.lens.device, dtype=torch.int32)
            binding.moda_kv_write_e4m3(self.pages, K, V, self.table, start=self.lens, n_new=more, bounds=self.bounds)
        except Exception:                                      # refused: nothing has happened
            self._enter(pages, taken=False)
            raise
        self._take(pages)
        self.lens += T if more is None else more
        self.lengths = [a + n for a, n in zip(self.lengths, count)]

    def read(self, T=None):
        """K, V bf16 [B,T,H_kv,d] of the first T (None: the longest sequence's) positions; zeros behind a sequence's last one."""
        T = self.longest if T is None else int(T)
        if T < 0:
            raise ValueError("T >= 0 required")
        if T == 0:
            return tuple(torch.empty((self.B, 0, self.H_kv, self.d), device=self.pages.device, dtype=torch.bfloat16) for _ in range(2))
        return binding.moda_kv_read_e4m3(self.pages, self.table, self.lens, T)

    def select(self, q, n_blocks: int, n_recent: int = 1, longest=None):
        """The blocks that a token attends to, [B, H_kv, n_blocks]: also for the layers or steps that use them again (``attend(..., index=...)``), until a sequence opens a
        block or its place changes hands: an older index does not have the newest positions, whatever ``n_recent`` was, and ``attend`` refuses it (this tensor
        itself: not a copy, and not one that a graph selects anew).  ``longest``: positions of a sequence that the call is for (None: of the longest now); ``max_len`` in a graph
        that is replayed while sequences grow."""
        if self.bounds is None:
            raise ValueError("this cache keeps no bounds")
        self.index = binding.moda_kv_select_blocks(q, self.bounds, self.table, self.lens, self.longest if longest is None else longest, n_blocks, n_recent)
        if not (self.index.is_cuda and torch.cuda.is_current_stream_capturing()):      # a graph's is made anew by every replay
            self.index.selected_for = (self._turns, *self._held())
        return self.index

    def _held(self):
        """Blocks of every place, and whose they are."""
        return [-(-n // 64) for n in self.lengths], list(self._turns)

    def attend(self, q, depth_kv_token, l, scale, n_blocks=None, n_recent: int = 1, index=None, O=None, LSE=None, workspace=None, longest=None):
        """The step of the token written last: O [B,H,d], LSE [B,H].  With ``n_blocks`` over so many selected blocks of 64 positions, with ``index`` over those.
        ``longest`` as for ``select``."""
        if n_blocks is not None:
            if index is not None:
                raise ValueError("n_blocks or index, not both")
            index = self.select(q, n_blocks, n_recent, longest)
        elif (made := getattr(index, "selected_for", None)) is not None:
            blocks, turns = self._held()
            if made[1] != blocks or (made[0] is self._turns and made[2] != turns):
                raise ValueError("the index is older than a block that a sequence has opened since, or than a sequence: select again")
        return binding.moda_attn_decode_e4m3(q, self.pages, self.table, self.lens, depth_kv_token, self.longest if longest is None else longest, l, scale, index=index, O=O, LSE=LSE,
                                             workspace=workspace)

    def release(self, b: int):
        """Sequence b has ended."""
        self._free.extend(reversed(self._owned[b]))
        self._owned[b] = []
        self._turns[b] += 1
        self.lengths[b] = 0
        self.lens[b] = 0
        self.table[b] = -1
