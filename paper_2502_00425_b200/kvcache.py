"""A paged key/value cache for one decoder block: the bookkeeping around the library's cache calls.

`PagedKVCache` owns the pool of pages, says which pages hold which sequence, and turns "these sequences get so many new
tokens" into the device arrays that mq_qk_norm_rope, mq_kv_attention, mq_kv_weights and mq_kv_evict take.  Lengths and
page lists are kept on the host (that is where a serving program decides); nothing here computes on keys or values.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

from . import binding as B


@dataclass
class CacheStep:
    """Device arrays for one step's new rows: the rows of sequence b are cu_q[b] .. cu_q[b + 1] - 1."""
    new: List[int]
    cu_q: torch.Tensor        # int32 [n_seq + 1]
    kv_len: torch.Tensor      # int32 [n_seq], the new keys included
    slots: torch.Tensor       # int64 [total], where each new row goes
    pos: torch.Tensor         # int32 [total], token positions in the order of the sequence
    total: int
    max_q: int

    def cu_q_host(self, b: int) -> int:
        return sum(self.new[:b])


class PagedKVCache:
    """n_seq sequences of up to max_len keys in n_pages pages of page_size tokens.  dtype bf16, or int8 with the static scales
    k_scale, v_scale (float32 [n_kv_heads]).  Its calls (and replays of graphs that captured them) follow one another in
    stream order: they share the workspaces, as they share the keys."""

    def __init__(self, n_seq: int, n_pages: int, max_len: int, n_kv_heads: int, head_dim: int, page_size: int = 64,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, device="cuda"):
        dtype = torch.int8 if k_scale is not None else torch.bfloat16
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        self.K, self.V = (torch.zeros(shape, dtype=dtype, device=device) for _ in range(2))
        self.handle = B.KVCache(self.K, self.V, k_scale, v_scale)
        self.n_seq, self.max_len, self.page_size = n_seq, max_len, page_size
        device = self.device = self.K.device      # (with its number: "cuda" would follow the current device)
        self.free = list(range(n_pages))[::-1]
        self.pages: List[List[int]] = [[] for _ in range(n_seq)]
        self.lengths = [0] * n_seq       # keys in the cache
        self.tokens = [0] * n_seq        # tokens seen: the next token's position (eviction does not change it)
        self.table = torch.full((n_seq, -(-max_len // page_size)), -1, dtype=torch.int32, device=device)
        self.weights: Optional[torch.Tensor] = None   # accumulated softmax weights, once track_weights() was called
        self.weights_status = torch.zeros(2, dtype=torch.int32, device=device)   # of every mq_kv_weights call
        self._ws = {}
        self._last: Optional[CacheStep] = None        # the step that undo() can take back

    def _take(self, n: int) -> List[int]:
        if n > len(self.free):
            raise RuntimeError(f"the cache has {len(self.free)} free pages, {n} are needed")
        return [self.free.pop() for _ in range(n)]

    def _give_back(self, pages: Sequence[int]):
        self.free += list(pages)[::-1]

    def _show(self, b: int, pages: Sequence[int]):
        row = torch.full((self.table.shape[1],), -1, dtype=torch.int32)
        row[:len(pages)] = torch.tensor(pages, dtype=torch.int32)
        self.table[b].copy_(row)

    def track_weights(self):
        """Keeps the softmax weight every key receives (mq_kv_weights), for evict(); called again, it starts over."""
        self.weights_status.zero_()
        self.weights = torch.zeros((self.n_seq, self.handle.n_kv_heads, self.max_len), device=self.device)

    def extend(self, new: Sequence[int]) -> CacheStep:
        """Room for new[b] tokens at the end of every sequence b, and the arrays of the step that brings them.  Where it raises,
        the cache is as it was."""
        assert len(new) == self.n_seq and min(new) >= 0
        ps, slots, pos, cu = self.page_size, [], [], [0]
        for b, n in enumerate(new):
            if self.lengths[b] + n > self.max_len:
                raise RuntimeError(f"sequence {b} would have {self.lengths[b] + n} keys, the cache was made for {self.max_len}")
        need = [max(0, -(-(self.lengths[b] + n) // ps) - len(self.pages[b])) for b, n in enumerate(new)]
        taken = self._take(sum(need))
        try:
            fresh, pages = list(taken), []
            lengths, tokens = [m + n for m, n in zip(self.lengths, new)], [m + n for m, n in zip(self.tokens, new)]
            for b, n in enumerate(new):
                pages.append(self.pages[b] + [fresh.pop() for _ in range(need[b])] if need[b] else self.pages[b])
                slots += [pages[b][j // ps] * ps + j % ps for j in range(self.lengths[b], lengths[b])]
                pos += range(self.tokens[b], tokens[b])
                cu.append(cu[-1] + n)
            dev = lambda v, t: torch.tensor(v, dtype=t).to(self.device)
            step = CacheStep(list(new), dev(cu, torch.int32), dev(lengths, torch.int32), dev(slots, torch.int64),
                             dev(pos, torch.int32), cu[-1], max(new))
            for b in range(self.n_seq):
                if need[b]:
                    self._show(b, pages[b])   # (entries behind a sequence's last key are not read)
        except BaseException:
            self._give_back(taken)
            raise
        self.pages, self.lengths, self.tokens, self._last = pages, lengths, tokens, step
        return step

    def undo(self, step: CacheStep):
        """Takes back the last extend(), for a step that could not be finished: its keys no longer count and its pages are free
        again.  Only the last step can be undone, and not behind an eviction.  (What attend() added to the tracked weights of
        earlier keys stays.)"""
        if step is not self._last:
            raise RuntimeError("only the last step can be undone")
        self._last = None
        for b in range(self.n_seq):
            self.lengths[b] -= step.new[b]
            self.tokens[b] -= step.new[b]
            keep = -(-self.lengths[b] // self.page_size)
            self.free += self.pages[b][keep:]
            del self.pages[b][keep:]

    def workspace(self, step: CacheStep, n_q_heads: int) -> torch.Tensor:
        """A workspace for the step, from a few sizes (powers of two) that are kept as long as the cache: a captured graph may
        hold any of them."""
        need = B.mq_kv_attention_workspace_bytes(self.n_seq, step.total, step.max_q, self.table.shape[1], n_q_heads, self.handle)
        size = max(1 << 16, 1 << (need - 1).bit_length())
        if size not in self._ws:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("run a step of this size once before capturing it: its workspace has to be made first")
            ws = torch.empty(size, dtype=torch.uint8, device=self.device)
            with torch.cuda.device(ws.device):
                B.mq_reset_device_status(ws)
            self._ws[size] = ws
        return self._ws[size]

    def attend(self, q: torch.Tensor, step: CacheStep, n_q_heads: int, perm: Optional[torch.Tensor] = None,
               scale: Optional[float] = None) -> torch.Tensor:
        """Attention of the step's rows over the cache (their keys and values are already stored); adds to the tracked weights."""
        o, lse = self.attention(q, step, n_q_heads, perm, scale)
        self.accumulate(q, lse, step, n_q_heads, perm, scale)
        return o

    def attention(self, q: torch.Tensor, step: CacheStep, n_q_heads: int, perm: Optional[torch.Tensor] = None,
                  scale: Optional[float] = None):
        """The attention alone: its result and the log-sum-exps."""
        o = torch.empty_like(q)
        lse = torch.empty((step.total, n_q_heads), device=q.device)
        B.mq_kv_attention(q, step.cu_q, step.kv_len, self.table, self.handle, n_q_heads, step.max_q, o, self.workspace(step, n_q_heads),
                          lse=lse, perm=perm, scale=scale)
        return o, lse

    def accumulate(self, q: torch.Tensor, lse: torch.Tensor, step: CacheStep, n_q_heads: int, perm: Optional[torch.Tensor] = None,
                   scale: Optional[float] = None):
        """Adds to the tracked weights, if there are any, what the step's rows gave (with attention()'s arguments)."""
        if self.weights is not None:
            B.mq_kv_weights(q, step.cu_q, step.kv_len, self.table, self.handle, n_q_heads, step.max_q, lse, self.weights,
                            w_in=self.weights, perm=perm, scale=scale, status=self.weights_status)

    def evict(self, budget: int, n_first: int, n_last: int) -> torch.Tensor:
        """Cuts every sequence to `budget` keys per head by the tracked weights; returns the kept indices (as mq_kv_evict's
        `kept`; entries behind a sequence's new length are -1).  The kept rows move to fresh pages, the old ones are freed.  The
        first n_first and last n_last keys are those of the cache: a chunk stored in AIFS order (forward_cached with images) has its
        visual tokens in front, so n_first keeps these rather than the text that stood before them."""
        if self.weights is None:
            raise RuntimeError("track_weights() first")
        if not self._ok(self.weights_status):   # (keys would be dropped for good by them)
            raise RuntimeError("the accumulated weights are not whole: a call that added to them has failed")
        ps = self.page_size
        after = [min(n, budget) for n in self.lengths]
        taken = self._take(sum(-(-n // ps) for n in after))
        try:
            pool = list(taken)
            fresh = [[pool.pop() for _ in range(-(-n // ps))] for n in after]
            table = torch.full((self.n_seq, max(1, -(-budget // ps))), -1, dtype=torch.int32)
            for b, p in enumerate(fresh):
                table[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
            kept = torch.full((self.n_seq, self.handle.n_kv_heads, budget), -1, dtype=torch.int32, device=self.device)
            new_len = torch.empty(self.n_seq, dtype=torch.int32, device=self.device)
            w_out = torch.zeros((self.n_seq, self.handle.n_kv_heads, budget), device=self.device)
            B.mq_kv_evict(self.handle, self.table, torch.tensor(self.lengths, dtype=torch.int32).to(self.device), self.weights, budget,
                          n_first, n_last, self.handle, table.to(self.device), kept, new_len, w_out=w_out)
        except BaseException:   # (refused, or no memory for its outputs: nothing has moved)
            self._give_back(taken)
            raise
        m = min(budget, self.max_len)
        self.weights.zero_()
        self.weights[:, :, :m] = w_out[:, :, :m]
        for b in range(self.n_seq):
            self.free += self.pages[b]
            self.pages[b], self.lengths[b] = fresh[b], after[b]
            self._show(b, fresh[b])
        self._last = None
        return kept

    def status_ok(self) -> bool:
        """Whether every attention and every accumulation of weights so far went through (waits for the current stream)."""
        return all(self._ok(s) for s in [*self._ws.values(), self.weights_status])

    @staticmethod
    def _ok(status: torch.Tensor) -> bool:
        with torch.cuda.device_of(status):      # (in the order of the calls, which run on its device's stream)
            return B.mq_last_device_status(status)[0] == B.MQ_OK
