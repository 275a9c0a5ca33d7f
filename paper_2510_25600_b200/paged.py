"""A paged K/V cache: the compressed prompts of several conversations, and the tokens that follow them.

    cache = PagedCache(...)
    pipe.run_device(q, k, v, pages=cache)           the prompt: what the selection keeps goes into the pages
    cache.advance(new)                              a step: room for each conversation's new tokens
        q = cache.append(layer, q, k, v, ...)       per layer: rotate, store
        o = cache.attend(layer, q)                  per layer: attention over all rows

This module owns the pools, hands out pages on the host and sequences calls of `binding`; it does no arithmetic of the method.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import binding as P


class PagedCache:
    """`n_layers` layers of `n_pages` pages of `page_size` rows, for `max_requests` conversations of up to `max_rows` rows each.  Conversation
    r is row r of `block_table` and `seq_lens`; one without rows is padding.  `dtype` torch.float8_e4m3fn holds rows in 8 bits, with
    scales [n_layers, n_kv_heads] (None: 1)."""

    def __init__(self, n_layers: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype, max_requests: int,
                 max_rows: int, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, device="cuda"):
        if min(n_layers, n_pages, page_size, n_kv_heads, head_dim, max_requests, max_rows) < 1:
            raise ValueError("a paged cache has at least one of everything")
        self.n_layers, self.n_pages, self.page_size, self.max_rows = n_layers, n_pages, page_size, max_rows
        self.k, self.v = (torch.empty((n_layers, n_pages, page_size, n_kv_heads, head_dim), dtype=dtype, device=device) for _ in "kv")
        self.k_scale, self.v_scale = k_scale, v_scale
        self.max_pages = -(-max_rows // page_size)
        # lengths and table: one buffer, so that a step's changes are one copy
        self._dev = torch.zeros(max_requests * (1 + self.max_pages), dtype=torch.int32, device=device)
        self.seq_lens = self._dev[:max_requests]
        self.block_table = self._dev[max_requests:].view(max_requests, self.max_pages)
        self.h_lens = np.zeros(max_requests, dtype=np.int32)
        self._pages: List[List[int]] = [[] for _ in range(max_requests)]
        self._free = list(range(n_pages - 1, -1, -1))
        self.on_gpu = self._dev.is_cuda
        # pinned copies, each with the event behind its last transfer
        self._ring = [[torch.zeros(self._dev.numel(), dtype=torch.int32, pin_memory=self.on_gpu), None] for _ in range(3)]
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def set_rows(self, rows: Sequence[int]) -> None:
        """Conversation r has rows[r] rows from now on (fewer than before give pages back); conversations past the end of `rows` keep
        theirs.  All or nothing: without enough free pages, RuntimeError, and nothing changes.  Not in a graph's capture, which would
        replay the lengths and pages of the capture."""
        if self.on_gpu and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the rows of a paged cache are set outside of a graph's capture")
        if len(rows) > len(self._pages) or any(n < 0 or n > self.max_rows for n in rows):
            raise ValueError(f"up to {len(self._pages)} conversations of 0 to {self.max_rows} rows, got {list(rows)}")
        want = [-(-int(n) // self.page_size) for n in rows]
        short = sum(w - len(p) for w, p in zip(want, self._pages)) - len(self._free)
        if short > 0:
            raise RuntimeError(f"the paged cache is {short} pages short")
        for r, w in enumerate(want):
            while len(self._pages[r]) > w:
                self._free.append(self._pages[r].pop())
        for r, w in enumerate(want):
            while len(self._pages[r]) < w:
                self._pages[r].append(self._free.pop())
        self.h_lens[:len(rows)] = rows
        self._upload()

    def advance(self, new: int | Sequence[int] = 1) -> None:
        """Room for `new` more rows: so many for every conversation that has rows, or as many for each as given."""
        if np.ndim(new) == 0:
            new = np.where(self.h_lens > 0, new, 0)
        self.set_rows(self.h_lens[:len(new)] + np.asarray(new))

    def release(self, r: int) -> None:
        """Conversation r is over: its pages are free for others from the next call on the stream on."""
        rows = self.h_lens.copy()
        rows[r] = 0
        self.set_rows(rows)

    def _upload(self) -> None:
        self._ring.append(self._ring.pop(0))
        slot = self._ring[0]
        if slot[1] is not None:
            slot[1].synchronize()
        host = slot[0].numpy()
        n = len(self._pages)
        host[:n] = self.h_lens
        table = host[n:].reshape(n, self.max_pages)
        for r, pages in enumerate(self._pages):
            table[r, :len(pages)] = pages
        self._dev.copy_(slot[0], non_blocking=True)
        if self.on_gpu:
            slot[1] = slot[1] or torch.cuda.Event()
            slot[1].record(torch.cuda.current_stream(self._dev.device))

    def store_prompt(self, k: torch.Tensor, v: torch.Tensor, idx: torch.Tensor, batch: P.Batch, budget: P.Budget) -> None:
        """The rows `idx` keeps of the prompts' K and V [n_layers,T,H_kv,d], behind what the first batch.n_req conversations have."""
        n = batch.n_req
        before = self.h_lens[:n].copy()
        self.set_rows(before + np.diff(budget.h_cu_kept))
        try:
            P.purekv_compact_paged(k, v, idx, batch, budget, self.k, self.v, self.block_table[:n], self.seq_lens[:n], k_scale=self.k_scale,
                                   v_scale=self.v_scale, status=self.status)
        except BaseException:
            self.set_rows(before)  # no rows without a prompt in them
            raise

    def _layer(self, layer: int) -> dict:
        return dict(k_scale=None if self.k_scale is None else self.k_scale[layer],
                    v_scale=None if self.v_scale is None else self.v_scale[layer], status=self.status)

    def append(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: Optional[torch.Tensor] = None,
               inv_freq: Optional[torch.Tensor] = None, sections: Optional[Sequence[int]] = None, interleaved: bool = False,
               cu_new: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The new tokens of a layer, after `advance`: rotates q and k and stores k and v.  Returns the rotated q.  Without `cu_new` there is
        a token for each of the first k.size(0) conversations."""
        n = k.size(0) if cu_new is None else cu_new.numel() - 1
        return P.purekv_append_paged(k, v, self.k[layer], self.v[layer], self.block_table[:n], self.seq_lens[:n], cu_new, q=q, q_out=q_out,
                                     positions=positions, inv_freq=inv_freq, sections=sections, interleaved=interleaved, **self._layer(layer))

    def attend(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               softmax_scale: float = 0.0, ws: Optional[torch.Tensor] = None, max_len: Optional[int] = None) -> torch.Tensor:
        """Attention of a new query per conversation (the first q.size(0) of them) over all their rows.  `max_len` sizes the launch: the
        longest conversation unless given, which a capture that is replayed later should do."""
        n = q.size(0)
        if max_len is None:
            max_len = int(self.h_lens[:n].max()) if n else 0
        return P.purekv_decode_paged(q, self.k[layer], self.v[layer], self.block_table[:n], self.seq_lens[:n], max_len=max_len, out=out, lse=lse,
                                     softmax_scale=softmax_scale, ws=ws, **self._layer(layer))

    def check_status(self) -> None:
        P.purekv_poll_status(self.status)
