"""K and V of a model's layers between a prompt's prefill and the tokens that follow it: the 8-bit paged
cache of every layer, one table and one pool of pages for all of them.

    kv = KVCache(n_layers, n_pages, n_kv_heads, max_seqs, max_tokens)
    granted = kv.reserve(counts)              # pages for the next rows, all layers
    o = kv.prefill(layer, seq, q, k, v)       # a prompt: sparse prefill, then K and V into the cache
    o = kv.prefill_packed(layer, row_ptr, q, k, v)   # or several (short) prompts at once: dense attention
    o = kv.attend(layer, row_ptr, q, k, v)    # a step: the rows' K and V in, then attention over all
    kv.advance(counts)                        # once all layers have run
    kv.evict(keep, cap)                       # long sequences cut to the tokens that had the most attention

With `rope` (C.make_rope) the calls turn q and k to the rows' positions first, which eviction does not change; with
`weights` they can add up the attention that each cached token gets, which eviction goes by.

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
    [max_seqs] (rows that each sequence may still take), pool (C.crisp_pool_init) and layers (a C.Cache each).  With rope or
    weights also pos int32 [max_seqs] (the position of each sequence's next token), with weights weights (float32 [max_seqs, H_kv,
    tokens] a layer) and held int32 [max_seqs] (tokens whose weights count).  The methods change them; they are there to be
    read."""

    def __init__(self, n_layers: int, n_pages: int, n_kv_heads: int, max_seqs: int, max_tokens: int, block: int = 64,
                 fmt: int = C.CACHE_E4M3, device="cuda", rope: Optional[C.CrispRopeTable] = None, weights: bool = False):
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
        self.rope = rope
        self.pos = self.held = self.weights = None
        if rope is not None or weights:
            self._pos = torch.zeros(max_seqs + 1, dtype=torch.int32, device=dev)  # the last row: of forks that are refused
            self.pos = self._pos[:-1]
        if weights:
            self._held = torch.zeros_like(self._pos)
            self._weights = [torch.empty(max_seqs + 1, n_kv_heads, self.table.shape[1] * block, device=dev) for _ in self.layers]
            self.held, self.weights = self._held[:-1], [w[:-1] for w in self._weights]

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

    def _turned(self, start: torch.Tensor, row_ptr: torch.Tensor, q: torch.Tensor, k: torch.Tensor):
        return (q, k) if self.rope is None else C.crisp_rope(self.rope, start, row_ptr, q, k)

    def _weigh(self, layer: int, table, seq_len, row_ptr, q, weights, held, softmax_scale: float) -> None:
        C.crisp_cache_weights(self.layers[layer], table, seq_len, row_ptr, q, weights, held, softmax_scale)

    def _need_weights(self) -> None:
        if self.weights is None:
            raise ValueError("a KVCache made with weights=True is needed")

    def prefill(self, layer: int, seq: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                params: Optional[C.CrispParams] = None, weigh: int = 0) -> torch.Tensor:
        """One layer of a prompt, sequence `seq` holding nothing yet and its pages reserved: sparse prefill
        attention over q [H_q, n, 128], k and v [H_kv, n, 128] as they are (turned, with rope), then k and v into the cache -> o.
        The attention that the prompt's tokens get from its last `weigh` rows is what they start with.  If the
        sequence holds tokens (attend() is for rows behind those) nothing is stored and o's first and last rows are NaN."""
        if not 0 <= seq < self.table.shape[0]:
            raise ValueError(f"sequence {seq} outside [0, {self.table.shape[0]})")
        n = k.shape[1]
        if weigh:
            self._need_weights()
            if not 0 < weigh <= n:
                raise ValueError(f"weigh {weigh} outside [0, {n}]")
        params = C.make_params() if params is None else params
        one = slice(seq, seq + 1)
        if self.rope is not None:
            q, k = self._turned(self.pos[one], self._all * n, q, k)
        o = C.crisp_prefill_attn(q, k, v, params)
        held = self.seq_len[seq] > 0
        o[:, ::max(n - 1, 1)].masked_fill_(held, math.nan)
        C.crisp_cache_append(self.layers[layer], torch.where(held, self._none, self._open[one]),
                             self.seq_len[one], self._all * n, k, v)
        if weigh:
            fits = ((self.seq_len[one] == 0) & (self.room[one] > 0)).int()  # otherwise no rows: nothing is written
            self._weigh(layer, self._open[one], fits * (n - weigh), self._all * (fits * weigh), q[:, n - weigh:],
                        self.weights[layer][one], torch.zeros_like(fits), params.softmax_scale)
        return o

    def prefill_packed(self, layer: int, row_ptr: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                       softmax_scale: float = 0.0, weigh: bool = False) -> torch.Tensor:
        """One layer of several prompts, rows row_ptr[s] .. row_ptr[s + 1] those of sequence s, which holds nothing yet: dense causal
        attention of each over itself, then k and v into the cache -> o.  With weigh, all their rows count (which for long prompts takes 10
        to 70 times what the attention takes; the last rows alone, as in prefill, take little).  If a
        sequence with rows holds tokens, nothing of it is stored and o's first row of it is NaN."""
        if weigh:
            self._need_weights()
        q, k = self._turned(self.pos, row_ptr, q, k)
        o = C.crisp_packed_attn(row_ptr, q, k, v, softmax_scale)
        n = q.shape[1]
        if n == 0:
            return o
        holds = self.seq_len > 0
        # a row that several sequences begin at (all but the last without rows) gets their sum: -0 changes nothing
        mark = torch.where(holds & (row_ptr[1:] > row_ptr[:-1]), math.nan, -0.0).to(o.dtype)
        o.index_add_(1, row_ptr[:-1].clamp(0, n - 1), mark[None, :, None].expand(o.shape[0], -1, o.shape[2]))
        table = torch.where(holds[:, None], self._none, self._open)
        C.crisp_cache_append(self.layers[layer], table, self.seq_len, row_ptr, k, v)
        if weigh:
            self._weigh(layer, table, self.seq_len, row_ptr, q, self.weights[layer], self.held, softmax_scale)
        return o

    def attend(self, layer: int, row_ptr: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
               softmax_scale: float = 0.0, ws: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None, weigh: bool = False) -> torch.Tensor:
        """One layer of a step: rows row_ptr[s] .. row_ptr[s + 1] of k and v behind sequence s's tokens, then q's
        rows over all of them -> o.  Rows of a sequence without room are not stored and get 0; of more rows than
        its room the ones behind it get no defined result.  With weigh the attention that each token gets is added to its
        weight (a sequence's weights are not defined after more rows than its room), at once: rows that advance() then does not take, or
        takes back later, leave in the weights of the tokens that stay what they added, and a layer's step that is run twice is
        added twice.  The workspace of that, up to 256 MB with the cache's size, is allocated in the call."""
        cache = self.layers[layer]
        if weigh:
            self._need_weights()
        q, k = self._turned(self.pos, row_ptr, q, k)
        C.crisp_cache_append(cache, self._open, self.seq_len, row_ptr, k, v)
        o = C.crisp_cache_attn(cache, self._open, self.seq_len, row_ptr, q, softmax_scale, ws, out)
        if weigh:
            self._weigh(layer, self._open, self.seq_len, row_ptr, q, self.weights[layer], self.held, softmax_scale)
        return o

    def advance(self, counts: torch.Tensor, weighed: bool = False) -> None:
        """The rows of a step, no more than were granted, count as held from here on (int32 [max_seqs]; negative to take
        tokens back, no more than are held: the sequence then takes no rows before reserve() has seen to it that none
        go into a page that a fork shares).  weighed: every layer's call of the step weighed them.  (The tokens of a step that
        was not weighed have weight 0 until one that is.)"""
        rows = self.room.clamp(max=counts)
        if self.pos is not None:
            self.pos.add_(rows.clamp(min=-self.seq_len))
        self.seq_len.add_(rows).clamp_(min=0)
        self.room.sub_(rows).masked_fill_(rows < 0, 0)
        if self.held is not None:
            torch.minimum(self.held, self.seq_len, out=self.held)
            if weighed:
                torch.where(rows > 0, self.seq_len, self.held, out=self.held)
        self._follow()

    def evict(self, keep: torch.Tensor, cap: int, sink: int = 4, recent: int = 64) -> torch.Tensor:
        """Between steps: sequences of more than keep[s] (int32 [max_seqs]; 0 or less, or above cap: stay as they are) tokens are cut to
        that many, in every layer and KV head the last `recent`, the first `sink`, and those that had the most weight -> the number
        of tokens kept, int32 [max_seqs], 0 where nothing was done: also where the free pages do not suffice, since what stays
        goes to pages of its own (a fork keeps what it shares).  Rows that were granted to a sequence that is cut and not
        taken are given back.  Positions go on as they were.  Tokens that advance() takes back later are the last places of each KV head: its
        `recent` ones, and where those do not suffice older tokens that stayed, in each head its own."""
        self._need_weights()
        if cap < 1:
            raise ValueError(f"cap {cap} must be positive")
        wanted = torch.where((keep < self.seq_len) & (keep <= cap), keep.clamp(min=0), torch.zeros_like(keep))
        slots = min(-(-cap // self.block), self.table.shape[1])
        new_table = torch.full_like(self.table[:, :slots], -1)
        count = C.crisp_pool_reserve(self.pool, self.block, new_table, torch.zeros_like(wanted), wanted)
        for cache, weights in zip(self.layers, self.weights):
            kept, _ = C.crisp_cache_keep(weights, self.held, self.seq_len, count, cap, sink, recent, weights)
            C.crisp_cache_gather(cache, self.table, kept, count, new_table)
        cut = count > 0
        ids = torch.where(cut, torch.arange(cut.shape[0], dtype=torch.int32, device=cut.device), self._none)
        C.crisp_pool_free(self.pool, self.table, self.seq_len, ids)
        self.table[:, :slots] = torch.where(cut[:, None], new_table, self.table[:, :slots])
        self.seq_len.add_(count)
        torch.where(cut, count, self.held, out=self.held)
        self.room.masked_fill_(cut, 0)
        self._follow()
        return count

    def fork(self, src: torch.Tensor, dst: torch.Tensor) -> torch.Tensor:
        """Empty sequences dst[i] become copies of src[i], sharing full pages -> copies int32 [n, 2], (-2, -2) where
        a fork was refused: that dst[i] is what it was, and rows that it is granted later are its first."""
        copies = C.crisp_pool_fork(self.pool, self.block, self.table, self.seq_len, src, dst)
        for cache in self.layers:
            C.crisp_cache_copy(cache, copies)
        if self.pos is not None:
            done, spare = copies[:, 0] != -2, self.table.shape[0]
            of, to = src.masked_fill(~done, spare).long(), dst.masked_fill(~done, spare).long()
            for t in [self._pos] + ([] if self.held is None else [self._held] + self._weights):
                t.index_copy_(0, to, t.index_select(0, of))
        return copies

    def free(self, ids: torch.Tensor) -> None:
        """Sequences ids[i] end."""
        C.crisp_pool_free(self.pool, self.table, self.seq_len, ids)
        gone = self.table[:, 0] < 0  # what was granted to a sequence is behind its first page
        for t in (self.room, self.pos, self.held):
            if t is not None:
                t.masked_fill_(gone, 0)
        self._follow()

    def compact(self) -> torch.Tensor:
        """All pages in use gathered at the front of every layer's cache -> the number of pages moved, int32 [1]."""
        moves, count = C.crisp_pool_compact(self.pool, self.table)
        self._follow()
        for cache in self.layers:
            C.crisp_cache_copy(cache, moves, count)
        return count
