"""The states of a target's linear-attention layers in a speculative round: the
buffers that ``spec_linear_attend`` and ``spec_linear_commit`` share, and a round's
calls on them; what ``paged.PagedCache`` is to the layers with keys and values.

    for layer in ...:
        states.attend(layer, q, k, v, log_decay, out, depth, row_offsets)    # outputs; the states stay
    spec_verify(...); spec_commit(...)
    for layer in ...:
        states.commit(layer, k, v, log_decay, accepted_len, depth, row_offsets)

and for a prompt, or a token that needs no verification, ``attend(..., update=True)``
alone.  Every step runs in libspec's kernels on the current stream (a fork also
moves a few integers); nothing waits for the device and no buffer changes its
place, so every call may be part of a captured graph.
"""
import torch

from . import MAX_LINEAR_ROWS, linear_workspace, spec_linear_attend, spec_linear_commit


class LinearStates:
    """States [key_dim, value_dim] of `layers` layers of `kv_heads` heads for up to
    `requests` requests and calls of up to `rows` rows each, zero at first.  A
    request has two slots of the pool, so that a fork never writes what it still
    reads.  `status` (int32 [1]) collects the calls' data errors."""

    def __init__(self, layers, q_heads, kv_heads, key_dim, value_dim, requests, rows, dtype=torch.bfloat16,
                 device="cuda"):
        if not 1 <= rows <= MAX_LINEAR_ROWS:
            raise ValueError(f"rows: 1 to {MAX_LINEAR_ROWS}")
        self.layers, self.B, self.rows = layers, requests, rows
        ints = dict(dtype=torch.int32, device=device)
        self._ws = linear_workspace(requests, rows - 1, q_heads, kv_heads, key_dim, value_dim, dtype, device)
        self.states = torch.zeros((layers, 2 * requests, kv_heads, key_dim, value_dim), device=device)
        self.slots = torch.arange(requests, **ints)            # where each request's states are
        self._spare = torch.arange(requests, 2 * requests, **ints)
        self.status = torch.zeros(1, **ints)
        # a call that only moves states: one row each, before position 0
        self._no_rows = torch.full((requests,), -1, dtype=torch.int64, device=device)
        self._no_k = torch.zeros((requests, kv_heads, key_dim), dtype=dtype, device=device)
        self._no_v = torch.zeros((requests, kv_heads, value_dim), dtype=dtype, device=device)
        self._no_decay = torch.zeros(kv_heads, device=device)

    def attend(self, layer, q, k, v, log_decay, out, depth=None, row_offsets=None, pos_base=None, update=False, K=None,
               scale=None, stream=None):
        """Outputs of the rows (requests of up to K + 1 rows; K = rows - 1 if None); with `update` their states too."""
        spec_linear_attend(q, k, v, log_decay, self.states, self.slots, self.slots if update else None, self.B,
                           self.rows - 1 if K is None else K, out, self._ws, row_offsets=row_offsets, depth=depth,
                           pos_base=pos_base, scale=scale, layer=layer, status=self.status, stream=stream)

    def commit(self, layer, k, v, log_decay, accepted_len=None, depth=None, row_offsets=None, pos_base=None, K=None,
               stream=None):
        """The first accepted_len + 1 rows (all if None) into the states."""
        spec_linear_commit(k, v, log_decay, self.states, self.slots, self.slots, accepted_len, self.B,
                           self.rows - 1 if K is None else K, self._ws, row_offsets=row_offsets, depth=depth,
                           pos_base=pos_base, layer=layer, status=self.status, stream=stream)

    def fork(self, parent, stream=None):
        """Request i becomes a copy of request parent[i] (int32 [B] on the device; -1: zero states, as for a request that
        begins; another that is no request's sets ERR_BAD_INPUT, and what its states are then is not said).  All
        requests' states move, those of requests that stay what they are among them."""
        if parent.shape != self.slots.shape:
            raise ValueError(f"parent: expected one of each of the {self.B} requests")
        with torch.cuda.stream(stream):
            start = self.slots[parent.clamp(0, self.B - 1).long()]
            start = start.masked_fill(parent < 0, -1).masked_fill((parent < -1) | (parent >= self.B), 2 * self.B)
            for layer in range(self.layers):
                spec_linear_commit(self._no_k, self._no_v, self._no_decay, self.states, start, self._spare, None, self.B,
                                   0, self._ws, pos_base=self._no_rows, layer=layer, status=self.status)
            old = self.slots.clone()
            self.slots.copy_(self._spare)
            self._spare.copy_(old)
