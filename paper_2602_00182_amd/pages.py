"""Bookkeeping of an 8-bit paged KV cache (host integers; the bytes move in det_kv8_copy_pages).

A pool of pages for all layers and a table [slots, max_pages] on the device that names the pages of each slot.  Slots may share pages (`fork`); a shared
page is copied before a slot may write into it (`reserve`); a page that no slot names is free again.  A slot may give up pages that its attention gave
little weight to (`evict`); they are holes in its table, the tokens behind them keep their positions, and they stay holes while the slot goes on.  The table
tensor keeps its address, so a captured graph sees what it holds at the replay."""
from __future__ import annotations

import contextlib
import heapq

import torch

from . import api


class OutOfPages(RuntimeError):
    """The pool has no free page left.  The call that raises it has changed nothing."""


class KVPages:
    def __init__(self, n_layers: int, n_pages: int, Hkv: int, n_slots: int, max_pages: int, D: int = 128, device="cuda"):
        if n_slots < 1 or max_pages < 1:
            raise ValueError("a page table needs slots and pages")
        self.pool = api.kv8_pool(n_layers, n_pages, Hkv, D, device)
        self.table = torch.full((n_slots, max_pages), -1, dtype=torch.int32, device=device)
        self._host = torch.full((n_slots, max_pages), -1, dtype=torch.int32)
        self._pages = [[] for _ in range(n_slots)]  # of each slot, in order
        self._forked = [0] * n_slots                # tokens of each slot up to which a fork shared its pages: it goes on behind them
        self._left = [None] * n_slots               # tokens at which a fork or a truncation left a slot that has not grown since
        self._refs = [0] * n_pages
        self._free = list(range(n_pages))           # a heap: the lowest page first
        self.version = 0                            # another one whenever the table has changed

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def _slots(self, *slots) -> None:
        """Refuses slots that are none; a negative index would name another slot from the end."""
        for slot in slots:
            if not 0 <= slot < len(self._pages):
                raise ValueError(f"slot {slot} of {len(self._pages)}")

    def pages(self, slot: int) -> list[int]:
        """The pages of a slot, in order; -1 where one was given up."""
        self._slots(slot)
        return list(self._pages[slot])

    def _copy(self, pairs, stream) -> None:  # with `stream` the current one: the pairs' tensors live in its memory
        if pairs:
            src, dst = (torch.tensor(x, dtype=torch.int32).to(self.pool.device) for x in zip(*pairs))
            api.det_kv8_copy_pages(self.pool, src, dst, stream)

    def _write_table(self) -> None:
        for slot, pages in enumerate(self._pages):
            self._host[slot].fill_(-1)
            self._host[slot, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        self.version += 1
        self.table.copy_(self._host)

    def _drop(self, page: int) -> None:
        if page < 0:
            return
        self._refs[page] -= 1
        if self._refs[page] == 0:
            heapq.heappush(self._free, page)

    def reserve(self, slots, lengths, write_from=None, stream=None) -> None:
        """Makes room for the first lengths[i] tokens of slots[i], and the pages from token write_from[i] on the slot's own: a shared page among
        them is copied where tokens in front of write_from[i] lie in it, else replaced.  Default: the slot is written behind the tokens that the longest of
        its forks shared (or that a truncation left of them), if lengths[i] reaches beyond them; a slot that writes further in front says so.
        Pages that a slot gave up get a page again where they begin at write_from[i] or behind, and none by default."""
        slots, lengths = list(slots), list(lengths)
        self._slots(*slots)
        if len(set(slots)) != len(slots) or len(lengths) != len(slots) or (write_from is not None and len(write_from) != len(slots)):
            raise ValueError("one length for each of several different slots")
        want, need = [], 0
        for i, (slot, length) in enumerate(zip(slots, lengths)):
            have, count = self._pages[slot], -(-length // api.KV8_PAGE)
            if length < 0 or count > self.table.shape[1]:
                raise ValueError("a length outside the page table")
            if write_from is not None:
                begin = int(write_from[i])
            else:
                begin = self._forked[slot] if length > self._forked[slot] else len(have) * api.KV8_PAGE
                left = self._left[slot]
                if left is not None and left < length and left % api.KV8_PAGE and have[left // api.KV8_PAGE] < 0:
                    raise ValueError("what is written next lies in a page that was given up")
            if begin < 0:
                raise ValueError("bad write_from")
            want.append((slot, begin, count, length))
        # how many references to each page go before its last sharer may keep it
        refs = dict()
        for slot, begin, count, _ in want:
            for i, page in enumerate(self._pages[slot][begin // api.KV8_PAGE:], begin // api.KV8_PAGE):
                if page < 0:
                    if write_from is None:
                        continue
                    if i * api.KV8_PAGE < begin:
                        raise ValueError("tokens in front of write_from lie in a page that was given up")
                    need += 1
                    continue
                r = refs.get(page, self._refs[page])
                if r > 1:
                    refs[page] = r - 1
                    need += 1
            need += max(0, count - len(self._pages[slot]))
        if need > len(self._free):
            raise OutOfPages(f"{need} pages wanted, {len(self._free)} free")
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            copies = []
            for slot, begin, count, length in want:
                pages = self._pages[slot]
                if self._left[slot] is not None and length > self._left[slot]:
                    self._left[slot] = None
                for i in range(begin // api.KV8_PAGE, len(pages)):
                    if pages[i] < 0 and write_from is None:
                        continue
                    if pages[i] < 0:
                        pages[i] = heapq.heappop(self._free)
                        self._refs[pages[i]] = 1
                    elif self._refs[pages[i]] > 1:
                        page = heapq.heappop(self._free)
                        if i * api.KV8_PAGE < begin:
                            copies.append((pages[i], page))
                        self._refs[pages[i]] -= 1
                        self._refs[page] = 1
                        pages[i] = page
                while len(pages) < count:
                    page = heapq.heappop(self._free)
                    self._refs[page] = 1
                    pages.append(page)
            self._copy(copies, stream)
            self._write_table()

    def fork(self, src: int, dsts, length: int, stream=None) -> None:
        """Each of the empty slots `dsts` shares the pages of the first `length` tokens of slot src.  Whoever writes into one of them reserves first."""
        count = -(-length // api.KV8_PAGE)
        dsts = list(dsts)
        self._slots(src, *dsts)
        if length < 0 or count > len(self._pages[src]) or len(set(dsts)) != len(dsts) or any(self._pages[s] for s in dsts) or src in dsts:
            raise ValueError("fork takes tokens that are there to different empty slots")
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            for s in dsts:
                self._pages[s] = self._pages[src][:count]
                self._forked[s] = self._left[s] = length
                self._forked[src] = max(self._forked[src], length)
                for page in self._pages[s]:
                    if page >= 0:
                        self._refs[page] += 1
            self._write_table()

    def truncate(self, slot: int, length: int, stream=None) -> None:
        """Gives back the pages behind the first `length` tokens of a slot (0: all of them)."""
        self._slots(slot)
        if length < 0:
            raise ValueError("a length outside the page table")
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            keep = -(-length // api.KV8_PAGE)
            for page in self._pages[slot][keep:]:
                self._drop(page)
            if length < len(self._pages[slot]) * api.KV8_PAGE:
                self._left[slot] = length
            del self._pages[slot][keep:]
            self._forked[slot] = min(self._forked[slot], length)
            self._write_table()

    def release(self, slot: int, stream=None) -> None:
        self.truncate(slot, 0, stream)

    def evict(self, weights, lengths, keep, first: int = 1, recent: int = 4, stream=None) -> list[list[int]]:
        """Each slot of lengths[s] tokens comes back to keep[s] pages: of those but its first `first` and last `recent` ones, it gives up the pages of least
        weight (det_kv8_pick_pages on weights [slots, max_pages], which attention with weights has added up; lengths and keep are int32 tensors on the
        device).  A page that other slots name stays theirs.  The weights are the caller's, who clears a slot's when it begins anew.  Waits for the device, and
        looks at every page of every slot on the host (64 slots of 512 pages: about 0.2 s).
        Returns the places in each slot's table that are holes now."""
        if recent < 1:
            raise ValueError("the page that is written goes on being there")
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            dropped = torch.empty(self.table.shape, dtype=torch.uint8, device=self.table.device)
            api.det_kv8_pick_pages(weights, self.table, self.pool.shape[1], lengths, keep, first, recent, dropped, stream)
            return self._give_up(dropped.cpu())

    def _give_up(self, dropped) -> list[list[int]]:
        gone = [[i for i in range(len(pages)) if dropped[slot, i] and pages[i] >= 0] for slot, pages in enumerate(self._pages)]
        for slot, places in enumerate(gone):
            for i in places:
                self._drop(self._pages[slot][i])
                self._pages[slot][i] = -1
        self._write_table()
        return gone

    def shared_tokens(self, slots) -> int:
        """How many of their first tokens the slots hold in the same pages (whole pages; ones that all have given up among them): what groups of rows say."""
        self._slots(*slots)
        pages = [self._pages[s] for s in slots]
        same = 0
        for of in zip(*pages):
            if any(p != of[0] for p in of):
                break
            same += 1
        return same * api.KV8_PAGE

    def compact(self, stream=None) -> int:
        """Moves the pages in use to the front of the pool; returns how many there are."""
        used = sum(1 for r in self._refs if r)
        high = [p for p in range(used, len(self._refs)) if self._refs[p]]
        low = [p for p in range(used) if not self._refs[p]]
        moved = dict(zip(high, low))  # as many of the one as of the other; no page is in both
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            self._copy(list(moved.items()), stream)
            for a, b in moved.items():
                self._refs[b], self._refs[a] = self._refs[a], 0
            self._pages = [[moved.get(p, p) for p in pages] for pages in self._pages]
            self._free = [p for p, r in enumerate(self._refs) if not r]
            self._write_table()
        return used
