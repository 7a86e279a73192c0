"""Multi-turn serving over the paged KV cache.

Sec. 2.3: with ISM a dialogue's KV cache is reused across turns, and every
turn extends it: the new query segment is prefilled against the cache (Eq. 5
first two cases), then the answer is generated token by token (third case,
f(j) = j). ``PagedKVCache`` runs those turns for many dialogues at once over
one pool of fixed-size pages, each call one launch sequence of the paged
entry points (``ops.prefill_paged``, ``ops.decode_paged``):

* ``prefill(slots, ..., seg_is_query=True)``: a new query segment;
* ``prefill(slots, ..., seg_is_query=False)``: a chunk of answer tokens, each
  row seeing the cache and the chunk's rows up to itself. A chunk of k
  drafted tokens is the same call: one launch verifies them (row r gives
  what decoding the r-th draft would give);
* ``decode(slots, ...)``: one answer token per dialogue;
* ``rollback(slot, length)``: drop rejected drafts (positions past
  ``length`` are no longer part of the dialogue; the next append overwrites
  them);
* ``release(slot)``: the dialogue ended; its pages return to the pool;
* ``fork(slot, new_slot)``: another continuation of the same dialogue (several
  answers to one turn). The two share every page; whichever appends first to
  a shared, partly filled page gets a copy of its own (``ops.copy_pages``);
* ``compact()``: moves the pages in use to the front of the pool.

With ``window`` (and ``sinks``) the attention is windowed
(``ops.prefill_paged_window``, ``ops.decode_paged_window``), and pages that lie
behind the window of every later token, and hold no sink, return to the pool
as the dialogue grows. A rollback to before such pages were freed is refused: to
answer a turn again, ``fork`` the dialogue before its answer is appended (the fork
keeps what it sees). Positions go on counting from the dialogue's first token, so
that it still ends at ``max_pages * page_size`` of them.

``PageAllocator`` is the host-side bookkeeping (no GPU): a free list of page
indices, the number of slots that hold each page, and each dialogue slot's
block table row and length.
"""

from __future__ import annotations

import contextlib

import numpy as np

from . import ops


class PoolExhausted(RuntimeError):
    """No free page is left for a dialogue's growth."""


class PageAllocator:
    """Free list over ``num_pages`` pages of ``page_size`` positions; slot b
    holds ``lens[b]`` positions in pages ``held[b]`` = ``table[b, :npages(b)]``
    (-1 in ``held``, 0 in ``table``: a page behind the window that was freed)."""

    def __init__(self, num_pages, page_size, slots, max_pages):
        if num_pages < 1 or page_size < 1 or slots < 1 or max_pages < 1:
            raise ValueError("num_pages, page_size, slots and max_pages must be positive")
        self.num_pages, self.page_size = int(num_pages), int(page_size)
        self.max_pages = int(max_pages)
        self._free = list(range(self.num_pages - 1, -1, -1))  # pop() -> lowest
        self.table = np.zeros((slots, self.max_pages), dtype=np.int32)
        self.held = [[] for _ in range(slots)]
        self.lens = np.zeros(slots, dtype=np.int64)
        self.refs = np.zeros(self.num_pages, dtype=np.int64)  # slots that hold each page
        # slot b's freed pages behind the window: held[b][first:end]
        self._trimmed = [(0, 0)] * slots

    @property
    def capacity(self):
        """Positions one slot can hold."""
        return self.max_pages * self.page_size

    def free_pages(self):
        return len(self._free)

    def reserve(self, slot, length):
        """Make pages cover positions [0, length) of ``slot``; all or nothing."""
        if length > self.capacity:
            raise ValueError(f"slot {slot}: {length} positions exceed the capacity "
                             f"{self.capacity} (max_pages x page_size)")
        held = self.held[slot]
        grow = -(-int(length) // self.page_size) - len(held)
        if grow > len(self._free):
            raise PoolExhausted(f"slot {slot} needs {grow} more pages, {len(self._free)} free")
        for _ in range(max(grow, 0)):
            page = self._free.pop()
            self.refs[page] = 1
            self.table[slot, len(held)] = page
            held.append(page)

    def _drop(self, page):
        self.refs[page] -= 1
        if self.refs[page] == 0:
            self._free.append(page)

    def rollback(self, slot, length, window=None):
        """Shorten ``slot`` to ``length`` positions; pages past them return.
        Under a window, not to where a later token would see a freed page."""
        if not 0 <= length <= self.lens[slot]:
            raise ValueError(f"slot {slot}: rollback to {length} outside [0, {self.lens[slot]}]")
        first, end = self._trimmed[slot]
        if end > first and length > first * self.page_size:
            if window is None or max(length - window + 1, 0) < end * self.page_size:
                raise ValueError(f"slot {slot}: rollback to {length} needs pages behind the "
                                 "window that were freed")
        else:
            self._trimmed[slot] = (0, 0)
        self.lens[slot] = length
        keep = -(-int(length) // self.page_size)
        held = self.held[slot]
        while len(held) > keep:
            page = held.pop()
            if page >= 0:
                self._drop(page)
            self.table[slot, len(held)] = 0

    def release(self, slot):
        self.rollback(slot, 0)

    def trim(self, slot, window, sinks):
        """Free the pages of ``slot`` that no token from position ``lens[slot]``
        on sees: wholly behind its window, without a sink. They are the last
        free pages to be used. Returns what ``untrim`` takes."""
        first = -(-int(sinks) // self.page_size)
        end = max(int(self.lens[slot]) - int(window) + 1, 0) // self.page_size
        before = self._trimmed[slot]
        done = max(first, before[1])
        pages = self.held[slot][done:end]
        for i, page in enumerate(pages, done):
            self.refs[page] -= 1
            self._put(slot, i, -1)
        if pages:
            self._trimmed[slot] = (first, done + len(pages))
            self._free[:0] = [page for page in pages if self.refs[page] == 0]
        return slot, done, pages, before

    def untrim(self, trimmed, lost=()):
        """Undo ``trim`` (its result), but for the pages in ``lost`` (their
        values are gone) and those before them."""
        slot, done, pages, before = trimmed
        for i in reversed(range(len(pages))):
            page = pages[i]
            if page in lost:
                return
            if self.refs[page] == 0:
                self._free.remove(page)
            self.refs[page] += 1
            self._put(slot, done + i, page)
            self._trimmed[slot] = (self._trimmed[slot][0], done + i) if i else before

    def fork(self, slot, new_slot):
        """``new_slot``, which must be empty, holds the same positions in the
        same pages."""
        if slot == new_slot or self.held[new_slot]:
            raise ValueError(f"fork: slot {new_slot} is not empty")
        keep = -(-int(self.lens[slot]) // self.page_size)
        pages = self.held[slot][:keep]
        for page in pages:
            if page >= 0:
                self.refs[page] += 1
        self.held[new_slot] = pages
        self.table[new_slot, :keep] = self.table[slot, :keep]
        self.lens[new_slot] = self.lens[slot]
        self._trimmed[new_slot] = self._trimmed[slot]

    def own_last(self, slot):
        """Before an append to ``slot``: if it goes on in a partly filled page
        that another slot holds too, put a free page in its place. Returns
        (old page, new page, positions to copy) or None."""
        used = int(self.lens[slot]) % self.page_size
        at = int(self.lens[slot]) // self.page_size
        if used == 0 or self.refs[self.held[slot][at]] == 1:
            return None
        if not self._free:
            raise PoolExhausted(f"slot {slot} needs a copy of a shared page, 0 free")
        old, new = self.held[slot][at], self._free.pop()
        self.refs[new] = 1
        self._put(slot, at, new)
        self._drop(old)
        return old, new, used

    def give_back(self, slot, copy):
        """Undo ``own_last`` (its result)."""
        if copy is not None:
            old, new, _ = copy
            self._put(slot, int(self.lens[slot]) // self.page_size, old)
            self.refs[old] += 1
            self._drop(new)

    def _put(self, slot, at, page):
        self.held[slot][at] = page
        self.table[slot, at] = max(page, 0)

    def compact(self):
        """Give the n pages in use the indices 0 .. n - 1. Returns (n, old
        indices, new indices) of the pages that move."""
        n, src, dst = self.moves()
        self.move(n, src, dst)
        return n, src, dst

    def moves(self):
        """What ``compact`` returns, with nothing changed."""
        used = np.flatnonzero(self.refs > 0)
        n = len(used)
        return n, used[used >= n], np.flatnonzero(self.refs[:n] == 0)

    def move(self, n, src, dst):
        """Give the pages src, of n in use, the indices dst."""
        new = np.arange(self.num_pages)
        new[src] = dst
        for slot, held in enumerate(self.held):
            for i, page in enumerate(held):
                if page >= n:
                    self._put(slot, i, int(new[page]))
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        self._free = list(range(self.num_pages - 1, n - 1, -1))


class PagedKVCache:
    """Device page pools, one block table row per dialogue slot, and the turn
    operations above. Pools are ``[num_pages, hkv, page_size, d]`` bf16. Each
    call uploads the block table rows and lengths of its slots (a small
    synchronous host-to-device copy): a reference loop, not a graph-captured
    one. ``window`` and ``sinks``: see ``ops.fwd_window``."""

    def __init__(self, num_pages, page_size, slots, max_pages, hkv, d, device="cuda",
                 window=None, sinks=0):
        import torch
        if window is not None and window < 1:
            raise ValueError(f"window {window} must be at least 1")
        if sinks < 0 or (sinks and window is None):
            raise ValueError(f"sinks {sinks} must be at least 0, and need a window")
        self.window, self.sinks = (None, 0) if window is None else ops._window(window, sinks)
        self.alloc = PageAllocator(num_pages, page_size, slots, max_pages)
        self.hkv, self.d, self.device = hkv, d, device
        shape = (num_pages, hkv, page_size, d)
        self.k_pages = torch.zeros(shape, dtype=torch.bfloat16, device=device)
        self.v_pages = torch.zeros(shape, dtype=torch.bfloat16, device=device)
        self._ws = None

    @property
    def lens(self):
        return self.alloc.lens

    def _reserve_all(self, slots, lengths):
        """Reserve pages for every slot or, if one request fails, for none
        (the pages reserved by this call go back to the pool). Returns the
        copies of shared pages that the appends need first."""
        return [copy for _, copy in self._reserved(slots, lengths) if copy is not None]

    def _reserved(self, slots, lengths):
        """``_reserve_all`` with each slot and its copy or None."""
        if len(set(slots)) != len(slots):
            raise ValueError("a slot appears twice in one call")
        done = []
        try:
            for s, n in zip(slots, lengths):
                self.alloc.reserve(s, n)
                done.append([s, None])
                done[-1][1] = self.alloc.own_last(s)
        except BaseException:
            self._give_back(done)
            raise
        return done

    def _give_back(self, done):
        for s, copy in reversed(done):
            self.alloc.give_back(s, copy)
            self._shrink(s)

    def _shrink(self, slot):
        """Pages reserved past the slot's length return."""
        held, keep = self.alloc.held[slot], -(-int(self.alloc.lens[slot]) // self.alloc.page_size)
        while len(held) > keep:
            self.alloc._drop(held.pop())
            self.alloc.table[slot, len(held)] = 0

    @contextlib.contextmanager
    def _appending(self, slots, new_lens):
        """Around an append of ``new_lens`` tokens to ``slots``: room for them,
        with the pages behind the window freed and shared pages that are written
        copied first. If any of it or the append is refused, the slots are as
        they were (but for pages behind the window that, the pool being short,
        a shared page was copied over: they stay freed)."""
        a, trimmed, done = self.alloc, [], []
        try:
            if self.window is not None:
                for s in slots:
                    trimmed.append(a.trim(s, self.window, self.sinks))
            done = self._reserved(slots, [a.lens[s] + n for s, n in zip(slots, new_lens)])
            self._copy([copy for _, copy in done if copy is not None])
            yield
        except BaseException:
            self._give_back(done)
            for t in reversed(trimmed):
                a.untrim(t, [copy[1] for _, copy in done if copy is not None])
            raise
        for s, n in zip(slots, new_lens):
            a.lens[s] += n

    def _copy(self, copies):
        import torch
        if copies:
            src, dst, tokens = (torch.tensor(x, dtype=torch.int32, device=self.device)
                                for x in zip(*copies))
            ops.copy_pages(self.k_pages, self.v_pages, src, dst, tokens)

    def _views(self, slots):
        import torch
        tab = torch.from_numpy(self.alloc.table[slots]).to(self.device)
        lens = torch.from_numpy(self.alloc.lens[slots].astype(np.int32)).to(self.device)
        return tab, lens

    def prefill(self, slots, q_new, k_new, v_new, new_lens, seg_is_query=True, scale=None):
        """New segment of ``new_lens[i]`` >= 1 tokens for each slot in
        ``slots`` (rows packed in slot order). Returns (o, lse)."""
        import torch
        slots = list(slots)
        new_lens = [int(n) for n in new_lens]
        if len(new_lens) != len(slots) or min(new_lens, default=1) < 1:
            raise ValueError("one new length >= 1 per slot")
        with self._appending(slots, new_lens):
            tab, lens = self._views(slots)
            cu = torch.tensor(np.concatenate([[0], np.cumsum(new_lens)]), dtype=torch.int32,
                              device=self.device)
            args = (q_new, k_new, v_new, self.k_pages, self.v_pages, tab, lens, cu, max(new_lens))
            if self.window is None:
                return ops.prefill_paged(*args, seg_is_query, scale)
            return ops.prefill_paged_window(*args, self.window, self.sinks, seg_is_query, scale)

    def decode(self, slots, q, k_new, v_new, scale=None, num_splits=0):
        """One answer token for each slot in ``slots``. Returns (o, lse)."""
        import torch
        slots = list(slots)
        with self._appending(slots, [1] * len(slots)):
            tab, lens = self._views(slots)
            sizes = (self.alloc.capacity, q.shape[1], self.hkv, self.d)
            if self.window is None:
                need = ops.workspace_size(ops.ISM_OP_DECODE, len(slots), 0, *sizes, num_splits)
            else:
                need = ops.window_workspace_size(ops.ISM_OP_DECODE, len(slots), 0, 0, *sizes,
                                                 self.window, self.sinks, num_splits)
            if self._ws is None or self._ws.numel() < need:
                self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
            args = (q, k_new, v_new, self.k_pages, self.v_pages, tab, lens)
            if self.window is None:
                return ops.decode_paged(*args, 0, scale, num_splits, workspace=self._ws)
            return ops.decode_paged_window(*args, self.window, self.sinks, 0, scale, num_splits,
                                           workspace=self._ws)

    def rollback(self, slot, length):
        self.alloc.rollback(slot, length, self.window)

    def release(self, slot):
        self.alloc.release(slot)

    def fork(self, slot, new_slot):
        """``new_slot`` (empty) continues the dialogue of ``slot`` on its own."""
        self.alloc.fork(slot, new_slot)

    def compact(self):
        """Move the pages in use to the front of the pools; returns their
        number. (Block tables of earlier calls are out of date then.)"""
        n, src, dst = self.alloc.moves()
        self._copy([(int(s), int(t), self.alloc.page_size) for s, t in zip(src, dst)])
        self.alloc.move(n, src, dst)
        return n
