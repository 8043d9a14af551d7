"""K and V of a model's layers between a prompt's prefill and the tokens that follow it: the 8-bit paged
cache of every layer, one table and one pool of pages for all of them.

    kv = KVCache(n_layers, n_pages, n_kv_heads, max_seqs, max_tokens)
    granted = kv.reserve(counts)              # pages for the next rows, all layers
    o = kv.prefill(layer, seq, q, k, v)       # a prompt: sparse prefill, then K and V into the cache
    o = kv.attend(layer, row_ptr, q, k, v)    # a step: the rows' K and V in, then attention over all
    kv.advance(counts)                        # once all layers have run

Everything stays on the GPU and is only enqueued, on the current stream; nothing waits for the device.  So that the
loop need not look at `granted`, rows that no reservation covers change nothing: they are not stored, what they
attend to is nothing (o is 0), and advance() does not count them.
"""
from __future__ import annotations

import math
from typing import Optional

import torch

from . import crisp as C


class KVCache:
    """table int32 [max_seqs, pages of max_tokens], seq_len int32 [max_seqs] (tokens that all layers hold), room int32
    [max_seqs] (rows that each sequence may still take), pool (C.crisp_pool_init) and layers (a C.Cache each).  The
    methods change them; they are there to be read."""

    def __init__(self, n_layers: int, n_pages: int, n_kv_heads: int, max_seqs: int, max_tokens: int, block: int = 64,
                 fmt: int = C.CACHE_E4M3, device="cuda"):
        if n_layers < 1 or max_seqs < 1 or max_tokens < 1:
            raise ValueError(f"n_layers {n_layers}, max_seqs {max_seqs} and max_tokens {max_tokens} must be positive")
        self.layers = [C.make_cache(n_pages, n_kv_heads, block, fmt, device) for _ in range(n_layers)]
        self.block = block
        self.pool = C.crisp_pool_init(n_pages, device)
        dev = self.pool.device
        self.table = torch.full((max_seqs, -(-max_tokens // block)), -1, dtype=torch.int32, device=dev)
        self.seq_len = torch.zeros(max_seqs, dtype=torch.int32, device=dev)
        self.room = torch.zeros_like(self.seq_len)
        # the table as rows go by it: sequences without room have no page there, so that theirs go nowhere and see nothing
        self._open, self._none = torch.full_like(self.table, -1), torch.full((), -1, dtype=torch.int32, device=dev)
        self._all = torch.arange(2, dtype=torch.int32, device=dev)  # times n: row_ptr of n rows of one sequence

    def reserve(self, counts: torch.Tensor) -> torch.Tensor:
        """Pages for counts[s] (int32 [max_seqs]) more tokens of each sequence -> granted: counts[s], or 0 where the
        free pages or the table do not suffice, or the rows would go into a page that a fork shares.  Such a sequence
        takes no rows until a later call grants it some; one that is granted rows may take them in several steps."""
        granted = C.crisp_pool_reserve(self.pool, self.block, self.table, self.seq_len, counts)
        torch.maximum(self.room, granted, out=self.room).masked_fill_(granted < counts, 0)
        self._follow()
        return granted

    def _follow(self) -> None:
        torch.where((self.room > 0)[:, None], self.table, self._none, out=self._open)

    def prefill(self, layer: int, seq: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                params: Optional[C.CrispParams] = None) -> torch.Tensor:
        """One layer of a prompt, sequence `seq` holding nothing yet and its pages reserved: sparse prefill
        attention over q [H_q, n, 128], k and v [H_kv, n, 128] as they are, then k and v into the cache -> o.  If the
        sequence holds tokens (attend() is for rows behind those) nothing is stored and o's first and last rows are NaN."""
        if not 0 <= seq < self.table.shape[0]:
            raise ValueError(f"sequence {seq} outside [0, {self.table.shape[0]})")
        o = C.crisp_prefill_attn(q, k, v, C.make_params() if params is None else params)
        n = k.shape[1]
        held = self.seq_len[seq] > 0
        o[:, ::max(n - 1, 1)].masked_fill_(held, math.nan)
        C.crisp_cache_append(self.layers[layer], torch.where(held, self._none, self._open[seq:seq + 1]),
                             self.seq_len[seq:seq + 1], self._all * n, k, v)
        return o

    def attend(self, layer: int, row_ptr: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               softmax_scale: float = 0.0, ws: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One layer of a step: rows row_ptr[s] .. row_ptr[s + 1] of k and v behind sequence s's tokens, then q's
        rows over all of them -> o.  Rows of a sequence without room are not stored and get 0; of more rows than
        its room the ones behind it get no defined result."""
        cache = self.layers[layer]
        C.crisp_cache_append(cache, self._open, self.seq_len, row_ptr, k, v)
        return C.crisp_cache_attn(cache, self._open, self.seq_len, row_ptr, q, softmax_scale, ws, out)

    def advance(self, counts: torch.Tensor) -> None:
        """The rows of a step, no more than were granted, count as held from here on (int32 [max_seqs]; negative to take
        tokens back, no more than are held: the sequence then takes no rows before reserve() has seen to it that none
        go into a page that a fork shares)."""
        rows = self.room.clamp(max=counts)
        self.seq_len.add_(rows).clamp_(min=0)
        self.room.sub_(rows).masked_fill_(rows < 0, 0)
        self._follow()

    def fork(self, src: torch.Tensor, dst: torch.Tensor) -> torch.Tensor:
        """Empty sequences dst[i] become copies of src[i], sharing full pages -> copies int32 [n, 2], (-2, -2) where
        a fork was refused: that dst[i] is what it was, and rows that it is granted later are its first."""
        copies = C.crisp_pool_fork(self.pool, self.block, self.table, self.seq_len, src, dst)
        for cache in self.layers:
            C.crisp_cache_copy(cache, copies)
        return copies

    def free(self, ids: torch.Tensor) -> None:
        """Sequences ids[i] end."""
        C.crisp_pool_free(self.pool, self.table, self.seq_len, ids)
        self.room.masked_fill_(self.table[:, 0] < 0, 0)  # what was granted to a sequence is behind its first page
        self._follow()

    def compact(self) -> torch.Tensor:
        """All pages in use gathered at the front of every layer's cache -> the number of pages moved, int32 [1]."""
        moves, count = C.crisp_pool_compact(self.pool, self.table)
        self._follow()
        for cache in self.layers:
            C.crisp_cache_copy(cache, moves, count)
        return count
