"""The 4-bit KV cache that decoding reads: what a prefill leaves, page by page.

The paper's modes apply to the prefill; decoding attends over the full KV cache (Section 4.2).  ``KVCache`` holds
the four tensors of that cache and calls the C entry points ``sa_cache_*`` on them; nothing is computed here.

A step of a model with some running sequences::

    new = add * cache.reserve(add)              # add: int32 [slots], the new tokens of each slot; none without room
    counts = new[slots]                         # slots: int32 [B], the sequences of the step
    for layer in range(layers):
        ...                                     # q, k, v: [B, H, T, d] of the new tokens
        cache.append(layer, k, v, slots, counts)
        y = cache.attend(layer, q, slots, counts)
    cache.advance(new)

Every call only enqueues work, so such a step can be captured into a CUDA graph; lengths, pages and who has room are
read when it runs.  A sequence without room stays as it was (its rows of y: undefined): try again after others
have left.  Rotary embedding comes before ``append`` and ``attend``: the tokens of a step in token-major layout are a
[1, H, B*T, d] view for ``sa_rope_apply``, with the table's rows gathered at the tokens' positions.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as sa


class KVCache:
    """Pages for ``slots`` sequences of up to ``max_tokens`` tokens each, shared by all layers' tables.

    ``pages``: pages of the pool (default: enough for every slot at its longest).  ``k_scale``, ``v_scale``:
    powers of two; values up to 2688 times them are held, blocks of 16 whose largest is below about 0.09 times
    them lose bits of their scale."""

    def __init__(self, layers: int, Hkv: int, d: int, slots: int, max_tokens: int, pages: Optional[int] = None,
                 page: int = 64, k_scale: float = 2.0 ** -4, v_scale: float = 2.0 ** -4, device="cuda"):
        if page not in (16, 32, 64, 128):
            raise ValueError("page must be 16, 32, 64 or 128 tokens")
        row = -(-max_tokens // page)
        pages = slots * row if pages is None else pages
        self.page, self.k_scale, self.v_scale = page, k_scale, v_scale
        self.pool = sa.sa_cache_pool(layers, pages, Hkv, page, d, device)
        self.table = torch.full((slots, row), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(slots, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.pool, self.table, self.lens, self.refs))

    def reserve(self, add: torch.Tensor) -> torch.Tensor:
        """Room for add[s] tokens (int32 [slots]) behind each slot's; int32 [slots]: 1 where it is there.  Slots
        without room (the pool or the slot's row is full) take no part in the step: counts and ``advance`` times the result."""
        return sa.sa_cache_reserve(self.pool, self.table, self.lens, self.refs, add, self.page)

    def append(self, layer: int, k, v, slots=None, counts=None):
        """Tokens without a page of their slot's own are left out and recorded (``sa_read_status``)."""
        sa.sa_cache_append(self.pool, self.table, self.lens, k, v, layer, slots, counts, self.k_scale, self.v_scale,
                           self.refs, self.page)

    def attend(self, layer: int, q, slots=None, counts=None, w=0, flags=sa.CAUSAL, scale=0.0, y=None, want_lse=False,
               lse=None):
        return sa.sa_cache_attend(self.pool, self.table, self.lens, q, layer, slots, counts, w, flags, scale,
                                  self.k_scale, self.v_scale, y, want_lse, lse, page=self.page)

    def read(self, layer: int, k, v, slots=None, starts=None, counts=None):
        """Tokens starts[b] + t (from 0) of a layer into k, v: what ``attend`` sees of them.  (The forward calls take as many
        queries as keys: a chunk goes on from a cached prefix through ``attend`` with flags 0, joined through lse with
        the chunk's attention to itself.)"""
        return sa.sa_cache_read(self.pool, self.table, k, v, layer, slots, starts, counts, self.k_scale, self.v_scale,
                                self.page)

    def advance(self, add: torch.Tensor):
        """The appended tokens count from now on (int32 [slots])."""
        self.lens.add_(add)

    def fork(self, parents: torch.Tensor, children: torch.Tensor):
        """Empty slots ``children`` go on from ``parents``; pages are shared until one of their holders writes."""
        sa.sa_cache_fork(self.table, self.lens, self.refs, parents, children, self.page)

    def free(self, slots: torch.Tensor):
        sa.sa_cache_free(self.table, self.lens, self.refs, slots)

    def compact(self) -> torch.Tensor:
        """Held pages to the front of the pool; their number, int32 [1] on the device."""
        return sa.sa_cache_compact(self.pool, self.table, self.refs)
