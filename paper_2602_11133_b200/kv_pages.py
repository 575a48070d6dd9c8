"""Host side of a paged key-value cache: which sequence has which pages of a pool.

Nothing here touches a device: calls return the page copies that have to be made (`jot.kv_copy_pages`) before the sequences
are used again, in the terms of that call -- no page twice among the targets, none both read and written -- and page tables and
slots as plain lists for tensors.  Pages can be shared: a fork costs no page until one side writes.
"""
from __future__ import annotations

import heapq
import operator
from typing import Dict, Hashable, Iterable, List, Sequence, Tuple

Copies = Tuple[List[int], List[int]]        # pages to read, pages to write


class OutOfPages(RuntimeError):
    """The pool has fewer free pages than a call needs; nothing has changed."""


class PagePool:
    def __init__(self, n_pages: int, page_size: int):
        n_pages, page_size = operator.index(n_pages), operator.index(page_size)
        if n_pages <= 0 or page_size <= 0:
            raise ValueError("PagePool: n_pages and page_size must be positive")
        self.n_pages, self.page_size = n_pages, page_size
        self._free = list(range(n_pages))               # a heap: low pages first, so that little has to move later
        self._users = [0] * n_pages                     # sequences that have the page
        self._pages: Dict[Hashable, List[int]] = {}
        self._length: Dict[Hashable, int] = {}

    # ---- what is there ------------------------------------------------------------------------------------------
    @property
    def free_pages(self) -> int:
        return len(self._free)

    def length(self, seq: Hashable) -> int:
        return self._length[seq]

    def pages(self, seq: Hashable) -> List[int]:
        return list(self._pages[seq])

    def table(self, seqs: Sequence[Hashable], width: int) -> List[List[int]]:
        """Rows of a page table, -1 behind a sequence's last page."""
        rows = [self._pages[s] for s in seqs]
        if any(len(r) > width for r in rows):
            raise ValueError(f"PagePool: a sequence has more than {width} pages")
        return [r + [-1] * (width - len(r)) for r in rows]

    def slots(self, seq: Hashable, positions: Iterable[int]) -> List[int]:
        """page * page_size + offset of each position; positions must lie inside the sequence."""
        pages, n, ps = self._pages[seq], self._length[seq], self.page_size
        out = []
        for p in positions:
            if not 0 <= p < n:
                raise ValueError(f"PagePool: position {p} outside a sequence of {n}")
            out.append(pages[p // ps] * ps + p % ps)
        return out

    # ---- sequences ----------------------------------------------------------------------------------------------
    def add(self, seq: Hashable, length: int) -> None:
        """A new sequence of `length` positions in pages of its own."""
        length = operator.index(length)
        if seq in self._pages:
            raise ValueError(f"PagePool: sequence {seq!r} is there already")
        self._pages[seq], self._length[seq] = [], 0
        try:
            self.resize(seq, length)
        except (OutOfPages, ValueError):
            del self._pages[seq], self._length[seq]
            raise

    def resize(self, seq: Hashable, length: int) -> None:
        """Pages for `length` positions: new ones behind the last, or the last ones given back.  (Positions that come into a
        page another sequence has, too, need own() before they are written.)"""
        length = operator.index(length)
        if length < 0:
            raise ValueError("PagePool: negative length")
        pages = self._pages[seq]
        need = (length + self.page_size - 1) // self.page_size
        if need > len(pages):
            pages.extend(self._take(need - len(pages)))
        while len(pages) > need:
            self._give(pages.pop())
        self._length[seq] = length

    def fork(self, seq: Hashable, child: Hashable) -> None:
        """`child` has what `seq` has, in the same pages: whoever is about to write calls own() first."""
        if child in self._pages:
            raise ValueError(f"PagePool: sequence {child!r} is there already")
        self._pages[child], self._length[child] = list(self._pages[seq]), self._length[seq]
        for p in self._pages[child]:
            self._users[p] += 1

    def own(self, seq: Hashable, lo: int, hi: int) -> Copies:
        """Pages of its own for positions [lo, hi) of `seq`: the copies to make before they are written."""
        if not 0 <= lo <= hi <= self._length[seq]:
            raise ValueError(f"PagePool: [{lo}, {hi}) outside a sequence of {self._length[seq]}")
        pages = self._pages[seq]
        shared = [] if lo == hi else [i for i in range(lo // self.page_size, (hi - 1) // self.page_size + 1) if self._users[pages[i]] > 1]
        src, dst = [pages[i] for i in shared], self._take(len(shared))
        for i, p in zip(shared, dst):
            self._users[pages[i]] -= 1
            pages[i] = p
        return src, dst

    def free(self, seq: Hashable) -> None:
        """Gives the sequence's pages back; those that another sequence has, too, stay with it."""
        for p in self._pages.pop(seq):
            self._give(p)
        del self._length[seq]

    def compact(self) -> Copies:
        """Moves the used pages to the pool's beginning: the copies to make before anything else, page tables to be made anew."""
        used = self.n_pages - len(self._free)
        holes = sorted(p for p in self._free if p < used)
        movers = [p for p in range(used, self.n_pages) if self._users[p]]
        to = dict(zip(movers, holes))
        for pages in self._pages.values():
            pages[:] = [to.get(p, p) for p in pages]
        for p, q in to.items():
            self._users[q], self._users[p] = self._users[p], 0
        self._free = list(range(used, self.n_pages))    # sorted: a heap
        return movers, holes

    # ---- pages --------------------------------------------------------------------------------------------------
    def _take(self, n: int) -> List[int]:
        if n > len(self._free):
            raise OutOfPages(f"PagePool: {n} pages wanted, {len(self._free)} free")
        out = [heapq.heappop(self._free) for _ in range(n)]
        for p in out:
            self._users[p] = 1
        return out

    def _give(self, page: int) -> None:
        self._users[page] -= 1
        if self._users[page] == 0:
            heapq.heappush(self._free, page)
