"""A paged key-value cache for the target forward of a speculative round: the
buffers that ``spec_attend`` and the ``spec_cache_*`` calls share, and a round's
calls on them.

Every step runs in libspec's kernels on the current stream (a fork also copies
the table); nothing here waits for the device, and no buffer changes its place,
so every call may be part of a captured graph.  A round, with the arrays that the
other entry points already have (``pos_base``, and ``row_offsets`` and ``depth``
from ``spec_allocate``):

    cache.reserve(pos_base, depth, row_offsets)           # pages for the rows
    for layer in ...:
        cache.append(layer, k_new, v_new, pos_base, depth, row_offsets)
        cache.attend(layer, q, pos_base, out, depth, row_offsets)
    spec_verify(...); spec_commit(...)
    cache.commit(pos_base, accepted_len)                  # rejected drafts' pages go back

A request idles in a round, with no page, no key and outputs of 0, if all of its
rows lie before position 0: at pos_base = -(drafts + 1) whatever its depth.

``cache.fork`` shares pages between requests (parallel samples, beams),
``cache.compact`` moves the live pages to the low end, and
``cache.commit(pos_base)`` with 0 gives a finished request's pages back.
"""
import torch

from . import (MAX_DRAFTS, attend_workspace, cache_workspace, spec_attend, spec_cache_append, spec_cache_compact,
               spec_cache_copy, spec_cache_fork, spec_cache_release, spec_cache_reserve)


class PagedCache:
    """Keys and values of `layers` layers in `pages` pages of `page_size`
    positions, for up to `requests` requests of up to `max_positions` positions
    and rounds of up to `drafts` + 1 rows each; `window` and `sinks` as in
    spec_attend.  `status` (int32 [1]) collects the calls' data errors."""

    def __init__(self, layers, pages, page_size, q_heads, kv_heads, head_dim, requests, max_positions, drafts,
                 dtype=torch.bfloat16, window=0, sinks=0, device="cuda"):
        if not 0 <= drafts <= MAX_DRAFTS:
            raise ValueError(f"drafts: 0 to {MAX_DRAFTS}")
        self.page_size, self.B, self.K = page_size, requests, drafts
        self.window, self.sinks = window, sinks
        max_pages = (max_positions + page_size - 1) // page_size
        ints = dict(dtype=torch.int32, device=device)
        shape = (layers, pages, page_size, kv_heads, head_dim)
        self.k = torch.empty(shape, dtype=dtype, device=device)
        self.v = torch.empty(shape, dtype=dtype, device=device)
        self.page_table = torch.full((requests, max_pages), -1, **ints)
        self.page_refs = torch.zeros(pages, **ints)
        self.status = torch.zeros(1, **ints)
        self.granted = torch.zeros(requests, **ints)
        self.page_map = torch.empty(pages, **ints)
        # pairs to copy: after a reservation at most one per slot that a round touches, after a compaction
        # at most half of the pages
        self._pairs = max(requests * (drafts // page_size + 2), max(1, pages // 2))
        self._src, self._dst = torch.empty(self._pairs, **ints), torch.empty(self._pairs, **ints)
        self._counts = torch.zeros(2, **ints)
        self._old_table = torch.empty_like(self.page_table)
        self._cache_ws = cache_workspace(requests, drafts, page_size, device)
        self._attend_ws = attend_workspace(requests, drafts, q_heads, kv_heads, head_dim, dtype, device)

    def reserve(self, pos_base, depth=None, row_offsets=None, stream=None):
        """Pages of their own for the rows at pos_base .. pos_base + depth of every request; shared pages that the
        rows reach are copied.  Returns the device tensor of 1s (granted) and 0s (the cache is full)."""
        spec_cache_reserve(self.page_table, self.page_refs, pos_base, self.B, self.K, self.page_size, self._src,
                           self._dst, self._counts, self.granted, self._cache_ws, row_offsets=row_offsets,
                           depth=depth, status=self.status, stream=stream)
        n = self.B * (self.K // self.page_size + 2)
        spec_cache_copy(self.k, self.v, self._src[:n], self._dst[:n], self._counts, status=self.status, stream=stream)
        return self.granted

    def append(self, layer, k_new, v_new, pos_base, depth=None, row_offsets=None, stream=None):
        """The rows' keys and values [R, kv_heads, head_dim] into their pages."""
        spec_cache_append(k_new, v_new, self.k, self.v, self.page_table, pos_base, self.B, self.K,
                          row_offsets=row_offsets, depth=depth, layer=layer, status=self.status, stream=stream)

    def attend(self, layer, q, pos_base, out, depth=None, row_offsets=None, scale=None, lse_out=None, stream=None):
        """Attention of the rows' queries [R, q_heads, head_dim] over their requests' positions, into `out`."""
        spec_attend(q, self.k, self.v, self.page_table, pos_base, self.B, self.K, out, self._attend_ws,
                    row_offsets=row_offsets, depth=depth, scale=scale, window=self.window, sinks=self.sinks,
                    lse_out=lse_out, layer=layer, status=self.status, stream=stream)

    def commit(self, pos_base, accepted_len=None, stream=None):
        """Gives back the pages past pos_base + accepted_len + 1 positions (past pos_base without accepted_len: 0
        ends a request), and those that the window has left behind."""
        spec_cache_release(self.page_table, self.page_refs, pos_base, self.page_size, accepted_len=accepted_len,
                           window=self.window, sinks=self.sinks, status=self.status, stream=stream)

    def fork(self, parent, stream=None):
        """Request i becomes a copy of request parent[i] (int32 [B] on the device; -1: empty), sharing its pages.  The
        new table takes the old one's place (the old one is copied aside first), so that captured calls find it."""
        with torch.cuda.stream(stream):
            self._old_table.copy_(self.page_table)
        spec_cache_fork(self._old_table, self.page_refs, parent, self.page_table, self.page_refs, status=self.status,
                        stream=stream)

    def compact(self, stream=None):
        """Moves the live pages to the lowest indices; page_map[old] is a page's new index."""
        n = max(1, self.page_refs.numel() // 2)
        spec_cache_compact(self.page_table, self.page_refs, self._src, self._dst, self.page_map, self._counts,
                           status=self.status, stream=stream)
        spec_cache_copy(self.k, self.v, self._src[:n], self._dst[:n], self._counts, status=self.status, stream=stream)
