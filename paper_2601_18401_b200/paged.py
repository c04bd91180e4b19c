"""A paged key/value cache with its tensors: what a serving program holds (``include/sla.h``, "paged key/value cache").

:class:`PagedCache` allocates the pool, the page table and the counts of one layer and forwards to the calls of the binding.
Lengths live on the device; nothing here waits for them.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B


class PagedCache:
    """Up to `n_slots` sequences of up to `max_tokens` tokens that share `n_pages` pages of `page_tokens` tokens."""

    def __init__(self, n_pages: int, n_slots: int, max_tokens: int, *, n_q_heads: int, n_kv_heads: int, head_dim: int = 128,
                 page_tokens: int = 64, dtype: torch.dtype = torch.bfloat16, device: int = 0, max_batch: Optional[int] = None,
                 max_new: int = 8192, params: Optional[B.sla_params_t] = None, share: Optional["PagedCache"] = None):
        """max_batch, max_new: the most sequences and new tokens of one call (they size the workspace); params: of the span decode
        step, when it is used.  share: the cache of another layer, whose table, lengths, counts, handle (a workspace for that layer's
        heads) and, where they are not given, params this one uses; pages, slots and lengths have to be the same."""
        dev = torch.device("cuda", device)
        width = -(-max_tokens // page_tokens)
        if share is not None and (share.k.shape[0], share.k.shape[2], *share.table.shape) != (n_pages, page_tokens, n_slots, width):
            raise ValueError("layers that share a table must have the same pages, page_tokens, slots and max_tokens")
        self.k = torch.empty(n_pages, n_kv_heads, page_tokens, head_dim, dtype=dtype, device=dev)
        self.v = torch.empty_like(self.k)
        if share is None:
            self.table = torch.full((n_slots, width), -1, dtype=torch.int32, device=dev)
            self.n_tokens = torch.zeros(n_slots, dtype=torch.int32, device=dev)
            self.ref = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        else:
            self.table, self.n_tokens, self.ref = share.table, share.n_tokens, share.ref
        self.cache = B.make_cache(self.k, self.v, self.table, self.n_tokens, self.ref)
        self.params = share.params if params is None and share is not None else params
        if share is None:
            need = B.sla_paged_workspace_bytes(self.cache, n_q_heads, max_batch or n_slots, max_new, params=params)
            if need == 0:
                raise ValueError("shapes or parameters the library does not support")
            self.handle = B.Handle(device, need)
        else:
            self.handle = share.handle

    def extend(self, cu_new=None, *, seq=None):
        """Room for the new tokens of every sequence -> position of each one's first, -1 where refused."""
        return B.sla_cache_extend(self.handle, self.cache, cu_new, seq=seq)

    def append(self, cu_new, first, k_new, v_new, *, seq=None):
        B.sla_cache_append(self.handle, self.cache, cu_new, first, k_new, v_new, seq=seq)

    def attend(self, q, cu_new=None, *, seq=None, max_new=None, window=0, softmax_scale=None, first=None):
        """Dense causal attention of the new tokens -> out, lse.  first: of `extend`; refused sequences then give 0 and -inf."""
        return B.sla_paged_attention(self.handle, q, self.cache, cu_new, seq=seq, max_new=max_new, window=window,
                                     softmax_scale=softmax_scale, first=first)

    def step(self, q_s, q, *, seq=None, max_tokens=None, first=None):
        """The span decode step of each sequence's last token -> out, lse, anchors, scores.  first: as for `attend`."""
        return B.sla_paged_decode_step(self.handle, q_s, q, self.cache, self.params, seq=seq, max_tokens=max_tokens, first=first)

    def fork(self, src, dst):
        return B.sla_cache_fork(self.handle, self.cache, src, dst)

    def release(self, seq):
        B.sla_cache_release(self.handle, self.cache, seq)

    def compact(self):
        return B.sla_cache_compact(self.handle, self.cache)

    def copy(self, pairs):
        """The page copies that `fork` or `compact` made on another layer's cache."""
        B.sla_cache_copy(self.handle, self.cache, pairs)

    def poll(self) -> int:
        """Waits and returns the status of the calls so far (SLA_OK, SLA_ERR_CACHE_FULL, ..)."""
        return B.sla_poll_status(self.handle)
