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

A layer whose queries and keys are still to be normalised and rotated stores
and turns them in one call, and sequences may start from others' tokens:

    q = cache.store_rotary(layer, rotary, pos, q, k, v, q_weight=wq, k_weight=wk)
    cache.fork(parent, fork_len)                       # more questions about the same images

With a ``window`` (and ``sinks``) every ``attend`` sees the latest tokens and the
first ones only, and ``trim`` also hands back the pages of what has left the window
(so it comes behind the attention of the tokens reserved last, in every layer).
A cache has one window: layers with another one, or with none, have a cache of their own.

Every step runs in libavtp.so on torch's current stream (torch copies the new
lengths over the old ones); nothing is read back to the host, and the state
lies in buffers that stay where they are, so the calls of a decode step can be
captured into a graph and replayed.  ``seq_len``, ``free_count``,
``block_table`` and ``free_pages`` are there to be read; ``reserve``, ``fork``
and ``trim`` change them.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import avtp as A


class PagedCache:
    """Pages of ``layers`` layers for ``requests`` sequences of at most
    ``max_pages`` pages each, out of ``n_pages`` in all.

    ``sharing``: sequences may be forked; ``trim`` then hands a page back when no
    sequence holds it any more.  ``window``, ``sinks``: what attention sees (this
    implies sharing; a row of the table still counts all of a sequence's tokens)."""

    def __init__(self, requests: int, n_pages: int, max_pages: int, Hkv: int, d: int,
                 page_size: int = 64, layers: int = 1, dtype=torch.bfloat16, device="cuda",
                 sharing: bool = False, window: Optional[int] = None, sinks: int = 0):
        if (window is not None and window < 1) or sinks < 0 or (window is None and sinks):
            raise ValueError("a window of 1 or more, and sinks of 0 or more with it, are needed")
        self.page_size = page_size
        self.window, self.sinks = window, sinks
        self.sharing = sharing or window is not None
        self.layers = [A.Pages.empty(n_pages, Hkv, page_size, d, dtype, device) for _ in range(layers)]
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        # lengths, the number of free pages and (sharing) the tokens that have left each
        # sequence's window side by side: one copy takes a call's results over
        size = requests + 1 + (requests if self.sharing else 0)
        self._state, self._after = ints(size), ints(size)
        self.seq_len, self.free_count = self._state[:requests], self._state[requests:requests + 1]
        if self.sharing:
            self.gone, self._gone_after = self._state[requests + 1:], self._after[requests + 1:]
            self._src, self._dst = ints(requests), ints(requests)
            self._ws = A.alloc_workspace(A.page_release_workspace_bytes(n_pages), device)
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

    def store_rotary(self, layer: int, rotary, pos: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                     v: torch.Tensor, q_weight: Optional[torch.Tensor] = None,
                     k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     slot_map: Optional[torch.Tensor] = None) -> torch.Tensor:
        """A layer's queries and keys of the tokens reserved last, normalised head
        by head (where a weight is given) and rotated by their positions (a
        ``Rotary``; pos [planes, N] or [N]); K and V go into the pages, the queries
        are returned."""
        if slot_map is None:
            slot_map = self.slots
        if slot_map is None:
            raise ValueError("no tokens have been reserved")
        return A.page_store_rotary(self.layers[layer], rotary, pos, q, k, v, slot_map, q_weight, k_weight, eps)

    def fork(self, parent: torch.Tensor, fork_len: Optional[torch.Tensor] = None,
             status: Optional[torch.Tensor] = None) -> None:
        """Every empty sequence b with parent[b] >= 0 gets the first fork_len[b] tokens
        of that sequence (all of them without a fork_len): their whole pages are shared, a
        last one filled in part is copied in every layer.  One that cannot be forked stays
        empty and flags FLAG_REFUSED, or FLAG_NO_PAGES, in ``status`` [B].  ``attend`` takes
        a fork's tokens from its next reservation on."""
        if not self.sharing:
            raise ValueError("a cache made with sharing=True is needed")
        B = self.seq_len.numel()
        if fork_len is None:
            fork_len = self.seq_len[parent.clamp(min=0, max=B - 1).long()]
        A.prepare_page_fork(self.page_size, parent, fork_len, self.seq_len, self.free_pages, self.free_count,
                            self.block_table, self._after[:B], self._after[B:], self._src, self._dst,
                            self.gone, self._gone_after, status)()
        for pages in self.layers:
            A.page_copy(pages, self._src, self._dst)
        self._state.copy_(self._after)

    def attend(self, layer: int, q: torch.Tensor, cu_q: torch.Tensor, softmax_scale: float,
               max_kv_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
               ws: Optional[torch.Tensor] = None):
        """The new tokens (the last cu_q[b+1] - cu_q[b] of each sequence, whose
        K and V are stored) over the layer's pages; returns (out, lse).  Queries
        of a request that got no place for them: out 0, lse -inf."""
        return A.page_attention(self.layers[layer], q, cu_q, self._seen, self.block_table,
                                softmax_scale, max_kv_len, out, lse, status, ws, window=self.window,
                                sinks=self.sinks)

    def trim(self, keep_len: torch.Tensor, status: Optional[torch.Tensor] = None) -> None:
        """Cut every sequence to its first keep_len tokens (0: it has ended), and with a
        window let go of what has left it, as the next token sees it: tokens that were
        reserved and still wait for ``attend`` see further back and come first.  With
        sharing, a cut inside a page that another sequence holds, or behind what the
        window has left, is refused: the sequence stays whole and flags FLAG_REFUSED in
        ``status`` [B]."""
        B = self.seq_len.numel()
        if self.sharing:
            A.prepare_page_release(self.page_size, keep_len, self.seq_len, self.block_table, self.free_pages,
                                   self.free_count, self._after[:B], self._after[B:], self._ws, self.window or 0,
                                   self.sinks, self.gone, self._gone_after, status)()
            torch.minimum(self._seen, self._after[:B], out=self._seen)
            self._state.copy_(self._after)
            return
        self._cut(keep_len, status)

    def _cut(self, keep_len: torch.Tensor, status: Optional[torch.Tensor] = None) -> None:
        """Lengths and pages only, every page as its sequence's own."""
        B = self.seq_len.numel()
        A.prepare_page_trim(self.page_size, keep_len, self.seq_len, self.block_table, self.free_pages,
                            self.free_count, self._after[:B], self._after[B:], status)()
        torch.minimum(self._seen, self._after[:B], out=self._seen)
        self._state.copy_(self._after)  # (of a window what is there already)

    def _mark(self):
        """What ``_take_back`` needs to undo the reservations that follow."""
        return self.seq_len.clone(), self._seen.clone(), self.slots

    def _take_back(self, mark) -> None:
        """Undo what was reserved since ``mark`` was made: the lengths are as they were
        and the pages are free again (the ones taken last on top of the stack).  What has
        left the windows stays as it is, so that tokens which wait for their attention
        keep the keys they see; pages taken since are no other sequence's, so a cut
        without a look at their holders is right for forks too."""
        seq_len, seen, self.slots = mark
        self._cut(seq_len)
        self._seen.copy_(seen)
