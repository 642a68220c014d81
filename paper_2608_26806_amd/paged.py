"""The K/V cache behind a pruning layer.

After a pruning layer every sequence has a length of its own, and a
progressive schedule (Sec. 3.3.2) shortens it again at the next one, so the
layers between two pruning layers share their lengths and no others do.  A
``PagedCache`` is the cache of such a group of layers: one block table, one
stack of free pages, and each layer's pages.

    cache.reserve(cu_out, dl.N_out)                    # room for the kept tokens
    cache.store(0, k, v, keep_idx=keep)                # their K and V, picked on the way
    cache.store(1, k1, v1)                             # the next layer's, of the kept tokens
    out, lse = cache.attend(layer, q, cu_q, scale)     # new tokens over the cache
    cache.trim(keep_len)                               # requests that ended, drafts taken back

Every step runs in libavtp.so on torch's current stream (torch copies the new
lengths over the old ones); nothing is read back to the host, and the state
lies in buffers that stay where they are, so the calls of a decode step can be
captured into a graph and replayed.  ``seq_len``, ``free_count``,
``block_table`` and ``free_pages`` are there to be read; ``reserve`` and
``trim`` change them.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import avtp as A


class PagedCache:
    """Pages of ``layers`` layers for ``requests`` sequences of at most
    ``max_pages`` pages each, out of ``n_pages`` in all."""

    def __init__(self, requests: int, n_pages: int, max_pages: int, Hkv: int, d: int,
                 page_size: int = 64, layers: int = 1, dtype=torch.bfloat16, device="cuda"):
        self.page_size = page_size
        self.layers = [A.Pages.empty(n_pages, Hkv, page_size, d, dtype, device) for _ in range(layers)]
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        # lengths and the number of free pages side by side: one copy takes a
        # call's results over
        self._state, self._after = ints(requests + 1), ints(requests + 1)
        self.seq_len, self.free_count = self._state[:requests], self._state[requests:]
        # the lengths as attention takes them: 0 for requests whose last new tokens
        # got no place, so that their queries see nothing
        self._seen = ints(requests)
        self.block_table = ints(requests, max_pages) - 1
        self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.free_count.fill_(n_pages)
        self.slots: Optional[torch.Tensor] = None  # of the tokens reserved last

    def reserve(self, cu_new: torch.Tensor, n_new: int, slot_map: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Room for cu_new[b+1] - cu_new[b] more tokens of every sequence, in
        every layer; returns their slots (n_new entries, -1 where a request got
        no place), which ``store`` takes by default.  A request without a place
        keeps its length, flags FLAG_NO_PAGES in ``status`` [B], and until a
        reservation gives it one ``attend`` gives its queries out 0 and lse -inf."""
        if slot_map is None:
            slot_map = torch.empty(n_new, dtype=torch.int32, device=cu_new.device)
        B = self.seq_len.numel()
        A.prepare_page_tables(self.page_size, cu_new, self.seq_len, self.free_pages, self.free_count,
                              self.block_table, slot_map, self._after[:B], self._after[B:], status,
                              kv_len=self._seen)()
        self._state.copy_(self._after)
        self.slots = slot_map
        return slot_map

    def store(self, layer: int, k: torch.Tensor, v: torch.Tensor, slot_map: Optional[torch.Tensor] = None,
              keep_idx: Optional[torch.Tensor] = None) -> None:
        """A layer's K and V of the tokens reserved last (or of ``slot_map``)."""
        if slot_map is None:
            slot_map = self.slots
        if slot_map is None:
            raise ValueError("no tokens have been reserved")
        A.page_store(self.layers[layer], k, v, slot_map, keep_idx)

    def attend(self, layer: int, q: torch.Tensor, cu_q: torch.Tensor, softmax_scale: float,
               max_kv_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None):
        """The new tokens (the last cu_q[b+1] - cu_q[b] of each sequence, whose
        K and V are stored) over the layer's pages; returns (out, lse).  Queries
        of a request that got no place for them: out 0, lse -inf."""
        return A.page_attention(self.layers[layer], q, cu_q, self._seen, self.block_table,
                                softmax_scale, max_kv_len, out, lse, status, ws)

    def trim(self, keep_len: torch.Tensor, status: Optional[torch.Tensor] = None) -> None:
        """Cut every sequence to its first keep_len tokens (0: it has ended)."""
        B = self.seq_len.numel()
        A.prepare_page_trim(self.page_size, keep_len, self.seq_len, self.block_table, self.free_pages,
                            self.free_count, self._after[:B], self._after[B:], status)()
        torch.minimum(self._seen, self._after[:B], out=self._seen)
        self._state.copy_(self._after)

    def _mark(self):
        """What ``_take_back`` needs to undo the reservations that follow."""
        return self.seq_len.clone(), self._seen.clone(), self.slots

    def _take_back(self, mark) -> None:
        """Undo what was reserved since ``mark`` was made: the lengths are as they were
        and the pages are free again (the ones taken last on top of the stack)."""
        seq_len, seen, self.slots = mark
        self.trim(seq_len)
        self._seen.copy_(seen)
