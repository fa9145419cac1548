"""A paged key/value cache for one decoder block: the bookkeeping around the library's cache calls.

`PagedKVCache` owns the pool of pages, says which pages hold which sequence, and turns "these sequences get so many new
tokens" into the device arrays that mq_qk_norm_rope, mq_kv_attention, mq_kv_weights and mq_kv_evict take.  Lengths and
page lists are kept on the host (that is where a serving program decides); nothing here computes on keys or values.

`DeviceKVCache` keeps lengths, page lists and free pages on the GPU instead (mq_kv_plan), so that whole steps can be captured in a graph
and replayed, lets sequences end and begin again, and shares prefixes between them (mq_kv_attention_shared).
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


def _workspace(cache, need: int) -> torch.Tensor:
    size = max(1 << 16, 1 << (need - 1).bit_length())
    if size not in cache._ws:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("run a step of this size once before capturing it: its workspace has to be made first")
        ws = torch.empty(size, dtype=torch.uint8, device=cache.device)
        with torch.cuda.device(ws.device):
            B.mq_reset_device_status(ws)
        cache._ws[size] = ws
    return cache._ws[size]


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
        return _workspace(self, B.mq_kv_attention_workspace_bytes(self.n_seq, step.total, step.max_q, self.table.shape[1], n_q_heads, self.handle))

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


class DeviceKVCache:
    """A paged cache for one decoder block whose bookkeeping lives on the GPU: every step (extend) is one call on the stream, nothing waits,
    and a captured step goes on from whatever the cache holds when it is replayed.  What cannot be done (no free page, a sequence
    beyond the pages that max_len needs) makes a step without rows, and shows in status_ok().  Arguments as PagedKVCache's; it accumulates no weights and
    evicts nothing.  Its calls, and replays of graphs that captured them, follow one another in stream order; a graph holds the groups of
    its time, and is captured anew after share() or release().

    shared_from: where a step's groups have at least so many numbers (keys and values, times channels) to read again, they are read once by
    mq_kv_attention_shared; below, the repeated reads come out of L2 faster than two lines of work and their join.  One new token each, bf16,
    shared against not: 28 / 4 heads of 128, 32 sequences over 2048 keys (65 million) 21.1 us against 21.7, over 3360 (106) 28.3 against 27.6, over
    4096 (130) 28.6 against 30.4, over 6144 (195) 31.0 against 38.6; 32 / 8 heads, 4 over 16384 (101) 28.5 against 31.9, 8 over 8192 (117) 28.5
    against 29.1, 64 over 1024 (132) 35.8 against 35.5, over 2048 (264) 36.7 against 51.6.  So between 65 and 130 million it depends on the sizes, and the
    choice is up to 6 % off.  Steps of several tokens gain earlier (four each, 28 / 4 heads, 32 sequences over 2048 keys: 37.7 against 50.6): where they are
    usual, half of this number is better."""

    def __init__(self, n_seq: int, n_pages: int, max_len: int, n_kv_heads: int, head_dim: int, page_size: int = 64,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, device="cuda", shared_from: int = 100_000_000):
        dtype = torch.int8 if k_scale is not None else torch.bfloat16
        self.shared_from = shared_from
        self.K, self.V = (torch.zeros((n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2))
        self.handle = B.KVCache(self.K, self.V, k_scale, v_scale)
        self.n_seq, self.max_len, self.page_size = n_seq, max_len, page_size
        device = self.device = self.K.device
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)
        self.table = ints(n_seq, -(-max_len // page_size)).fill_(-1)
        self.kv_len, self.seen, self.borrowed, self.shared_len = (ints(n_seq) for _ in range(4))
        self.leader = torch.arange(n_seq, dtype=torch.int32, device=device)
        self.free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
        self.n_free = torch.full((1,), n_pages, dtype=torch.int32, device=device)
        self.plan_status = ints(2)
        self.state = B.KVState(self.kv_len, self.seen, self.table, self.free, self.n_free, page_size, borrowed=self.borrowed)
        self.leaders = list(range(n_seq))   # whose pages a sequence begins with: its own, or those it borrows
        self._heads = list(range(n_seq))    # as `leader` says: of every sequence, the first of those that are read together
        self._ended = [False] * n_seq       # released, and without rows since
        self._lent = [0] * n_seq            # keys that others have from a sequence, or that it has from another
        self._ws = {}
        self._numbers = {}                  # small device arrays, by what they hold
        self._captured = set()              # those that a graph may hold
        self._last: Optional[CacheStep] = None

    def _ints(self, values: Sequence[int]) -> torch.Tensor:
        key = tuple(values)
        capturing = torch.cuda.is_current_stream_capturing()
        if key not in self._numbers:
            if capturing:
                raise RuntimeError("make a step of these sizes once before capturing it: its arrays have to be made first")
            if len(self._numbers) >= 256:
                self._numbers = {k: v for k, v in self._numbers.items() if k in self._captured}
            # (from pinned memory, which torch does not hand out again before the copy is done: a copy from other memory waits for all that is queued)
            pinned = torch.tensor(key, dtype=torch.int32, pin_memory=self.device.type == "cuda")
            self._numbers[key] = pinned.to(self.device, non_blocking=True)
        numbers = self._numbers[key]
        if capturing:
            self._captured.add(key)
        elif numbers.is_cuda:               # (it may be dropped while a stream that did not make it has yet to read it)
            numbers.record_stream(torch.cuda.current_stream(self.device))
        return numbers

    def _group(self, ended: List[bool]):
        """Neighbours that begin with the same pages are read together, whichever of them is the first (the pages are in every one's list); one that has
        ended parts them only when it gets rows again, as a sequence of its own."""
        heads, last = list(range(self.n_seq)), None
        for b in range(self.n_seq):
            if ended[b]:
                continue
            if last is not None and self.leaders[b] == self.leaders[last]:
                heads[last + 1:b + 1] = [heads[last]] * (b - last)
            last = b
        if heads != self._heads:
            if torch.cuda.is_current_stream_capturing():   # (the host would know of groups that the GPU has only once the graph is replayed)
                raise RuntimeError("make a step of these sizes once before capturing it: a sequence begins again in it")
            self.leader.copy_(self._ints(heads))
            self._heads = heads
        self._ended = ended

    def _plan(self, new: torch.Tensor, keep: Optional[torch.Tensor], rows: int):
        cu = torch.empty(self.n_seq + 1, dtype=torch.int32, device=self.device)
        slots, pos = (torch.empty(rows, dtype=t, device=self.device) for t in (torch.int64, torch.int32))
        B.mq_kv_plan(self.state, new, cu, slots, pos, self.plan_status, keep=keep)
        return cu, slots, pos

    def extend(self, new: Sequence[int], keep: Optional[Sequence[int]] = None) -> CacheStep:
        """Room for new[b] tokens at the end of every sequence b, of which keep[b] keys stay (None: all of every sequence; 0 ends one, and what
        it gets is a new one; what is lent or borrowed stays until release()), and the arrays of the step that brings them."""
        assert len(new) == self.n_seq and min(new) >= 0
        if keep is not None and any(k < n for k, n in zip(keep, self._lent)):
            raise RuntimeError("a sequence keeps what others borrow from it, and what it has borrowed")
        if any(n and e for n, e in zip(new, self._ended)):
            self._group([e and not n for n, e in zip(new, self._ended)])
        total = sum(new)
        cu, slots, pos = self._plan(self._ints(new), None if keep is None else self._ints(keep), total)
        self._last = CacheStep(list(new), cu, self.kv_len, slots, pos, total, max(new))
        return self._last

    def undo(self, step: CacheStep):
        """Takes back the last extend(): its rows no longer count and their pages are free again."""
        if step is not self._last:
            raise RuntimeError("only the last step can be undone")
        self._last = None
        got = step.cu_q[1:] - step.cu_q[:-1]          # (none, if the step could not be made)
        self._plan(self._ints([0] * self.n_seq), self.kv_len - got, 0)

    def share(self, src: int, first: int, count: int) -> int:
        """Sequences first .. first + count - 1, which are empty, begin with the whole pages of sequence src, which stay its own (it cannot be
        released before them).  They stand behind src or its other borrowers.  Returns the number of keys they have then; what src has
        behind its last whole page they get by extend().  Waits for the stream."""
        to = range(first, first + count)
        if self.leaders[src] != src or first <= src or any(self.leaders[b] != src for b in range(src, first)):
            raise RuntimeError("borrowers stand directly behind the sequence they borrow from")
        if count < 1 or first + count > self.n_seq or any(self.leaders[b] != b for b in to):
            raise RuntimeError("not that many sequences of their own")
        lengths = self.lengths()
        if any(lengths[b] for b in to) or any(b in self.leaders[:b] + self.leaders[b + 1:] for b in to):
            raise RuntimeError("a sequence that borrows pages is empty, and lends none")
        pages = lengths[src] // self.page_size
        rows = slice(first, first + count)
        self.table[rows] = self.table[src]
        for array, value in ((self.borrowed, pages), (self.kv_len, pages * self.page_size), (self.shared_len, pages * self.page_size)):
            array[rows] = value
        self.seen[rows] = self.seen[src] - (lengths[src] - pages * self.page_size)
        self.shared_len[src] = 1 << 30                # (as far as the others go)
        self.leaders[first:first + count] = [src] * count
        self._lent[src] = max(self._lent[src], pages * self.page_size)
        self._lent[first:first + count] = [pages * self.page_size] * count
        self._group([e and b not in to for b, e in enumerate(self._ended)])
        self._last = None
        return pages * self.page_size

    def release(self, sequences: Sequence[int]):
        """Ends sequences: their own pages are free again.  Not while a stream is captured."""
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("sequences are not released while a stream is captured")
        if any(not 0 <= b < self.n_seq for b in sequences):
            raise RuntimeError("no such sequence")
        left = [l for b, l in enumerate(self.leaders) if l != b and b not in sequences]
        if any(b in left for b in sequences):
            raise RuntimeError("a sequence cannot end before those that borrow its pages")
        self._plan(self._ints([0] * self.n_seq), self._ints([0 if b in sequences else 1 << 30 for b in range(self.n_seq)]), 0)
        for b in sequences:
            self.leaders[b] = b
            self._lent[b] = 0
        for b in range(self.n_seq):
            if self.leaders[b] == b and b not in self.leaders[:b] + self.leaders[b + 1:]:
                self._lent[b] = 0
        self._group([e or b in sequences for b, e in enumerate(self._ended)])
        for b in sequences:
            self.shared_len[b] = 0
        self._last = None

    def lengths(self) -> List[int]:
        """Keys of every sequence (waits for the stream)."""
        return self.kv_len.tolist()

    def _shares(self, step: CacheStep) -> bool:
        if self.n_seq > 1024 or not any(self._lent):   # (the shared form's limit; every sequence's pages are in its own row as well)
            return False
        rows, keys = {}, {}
        for b, h in enumerate(self._heads):
            if step.new[b]:
                rows[h] = rows.get(h, 0) + 1
                if self.leaders[b] != b:
                    keys[h] = min(keys.get(h, self.max_len), self._lent[b])
        numbers = 2 * self.handle.n_kv_heads * self.handle.head_dim
        return any(rows[h] > 1 for h in keys) and sum((rows[h] - 1) * k for h, k in keys.items()) * numbers >= self.shared_from

    def workspace(self, step: CacheStep, n_q_heads: int) -> torch.Tensor:
        """As PagedKVCache.workspace()."""
        return self._attention_workspace(step, n_q_heads, self._shares(step))

    def _attention_workspace(self, step: CacheStep, n_q_heads: int, shares: bool) -> torch.Tensor:
        size_of = B.mq_kv_attention_shared_workspace_bytes if shares else B.mq_kv_attention_workspace_bytes
        return _workspace(self, size_of(self.n_seq, step.total, step.max_q, self.table.shape[1], n_q_heads, self.handle))

    def attention(self, q: torch.Tensor, step: CacheStep, n_q_heads: int, perm: Optional[torch.Tensor] = None,
                  scale: Optional[float] = None):
        """Attention of the step's rows over the cache (their keys and values are already stored), what a group shares being read once for
        all of it where that is faster: the result and the log-sum-exps."""
        o = torch.empty_like(q)
        lse = torch.empty((step.total, n_q_heads), device=q.device)
        shares = self._shares(step)
        ws = self._attention_workspace(step, n_q_heads, shares)
        if shares:
            B.mq_kv_attention_shared(q, step.cu_q, step.kv_len, self.table, self.leader, self.shared_len, self.handle, n_q_heads, step.max_q, o,
                                     ws, lse=lse, perm=perm, scale=scale)
        else:
            B.mq_kv_attention(q, step.cu_q, step.kv_len, self.table, self.handle, n_q_heads, step.max_q, o, ws, lse=lse, perm=perm, scale=scale)
        return o, lse

    def accumulate(self, q, lse, step, n_q_heads, perm=None, scale=None):
        """(This cache keeps no weights.)"""

    def status_ok(self) -> bool:
        """Whether every step could be made and every attention went through (waits for the current stream)."""
        return all(PagedKVCache._ok(s) for s in [*self._ws.values(), self.plan_status])
