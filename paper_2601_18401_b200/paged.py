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
                 max_new: Optional[int] = None, params: Optional[B.sla_params_t] = None, share: Optional["PagedCache"] = None,
                 four_bits: bool = False):
        """four_bits: keys and values are rounded to four bits as they are appended (dtype is then that of the calls' tensors), and there is
        no span decode step.  max_batch, max_new: the most sequences and new tokens of one call (they size the workspace; n_slots and 8192, or those of share, where
        they are not given); params: of the span decode step, when it is used.  share: the cache of another layer, whose table, lengths,
        counts and, where they are not given, params this one uses, and a handle of the layers that share it unless this layer's calls need
        a larger workspace than they have; pages, slots and lengths have to be the same."""
        dev = torch.device("cuda", device)
        width = -(-max_tokens // page_tokens)
        if share is not None and (share.k.shape[0], share.cache.page_tokens, *share.table.shape) != (n_pages, page_tokens, n_slots, width):
            raise ValueError("layers that share a table must have the same pages, page_tokens, slots and max_tokens")
        if four_bits and params is not None:
            raise ValueError("no span decode step over a cache in four bits: params must be None")
        if four_bits:
            self.k = torch.empty(n_pages, n_kv_heads, B.q4_plane_bytes(page_tokens, head_dim), dtype=torch.uint8, device=dev)
        else:
            self.k = torch.empty(n_pages, n_kv_heads, page_tokens, head_dim, dtype=dtype, device=dev)
        self.v = torch.empty_like(self.k)
        if share is None:
            self.table = torch.full((n_slots, width), -1, dtype=torch.int32, device=dev)
            self.n_tokens = torch.zeros(n_slots, dtype=torch.int32, device=dev)
            self.ref = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        else:
            self.table, self.n_tokens, self.ref = share.table, share.n_tokens, share.ref
        if four_bits:
            self.cache = B.make_cache_q4(self.k, self.v, self.table, self.n_tokens, self.ref, page_tokens=page_tokens, head_dim=head_dim,
                                         dtype=dtype)
        else:
            self.cache = B.make_cache(self.k, self.v, self.table, self.n_tokens, self.ref)
        self.params = share.params if params is None and share is not None else params
        self.max_batch = max_batch or (n_slots if share is None else share.max_batch)
        self.max_new = max_new if max_new is not None else 8192 if share is None else share.max_new
        need = B.sla_paged_workspace_bytes(self.cache, n_q_heads, self.max_batch, self.max_new, params=None if four_bits else self.params)
        if share is None and need == 0:
            raise ValueError("shapes or parameters the library does not support")
        self.handles = [] if share is None else share.handles   # of the layers that share the table
        enough = [] if share is None else [h for h in (share.handle, *share.handles) if h.workspace_bytes >= need]
        if not enough:
            enough = [B.Handle(device, need)]
            self.handles += enough
        self.handle = enough[0]

    def extend(self, cu_new=None, *, seq=None):
        """Room for the new tokens of every sequence -> position of each one's first, -1 where refused."""
        return B.sla_cache_extend(self.handle, self.cache, cu_new, seq=seq)

    def append(self, cu_new, first, k_new, v_new, *, seq=None):
        B.sla_cache_append(self.handle, self.cache, cu_new, first, k_new, v_new, seq=seq)

    def read(self, cu_new=None, first=None, *, n_new=None, seq=None, k_out=None, v_out=None):
        """Keys and values of the positions first[x] .. (None: 0 ..) of the sequences -> k, v [n_new, Hkv, D]."""
        return B.sla_cache_read(self.handle, self.cache, cu_new, first, n_new=n_new, seq=seq, k_out=k_out, v_out=v_out)

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
        """Waits and returns the status of the calls so far (SLA_OK, SLA_ERR_CACHE_FULL, ..), those of the layers that share the table included;
        where several have something to report, the next poll returns the next."""
        for handle in self.handles:
            status = B.sla_poll_status(handle)
            if status != B.SLA_OK:
                return status
        return B.SLA_OK
