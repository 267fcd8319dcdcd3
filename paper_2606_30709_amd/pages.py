"""Sequences in the pages of a cache: allocation, sharing, copying, moving.

``PageBook`` is the host's part: which page holds which chunk of which
sequence, how many sequences share a page, which pages are free.  It touches no
device.  ``PagedCache`` keeps a pool and a page table on the GPU in step with
it, with ``hga_copy_pages`` for what has to move, whichever device is current.

A page is shared by the sequences that were forked from one another until one
of them appends to it; that one then gets a copy of its own.  All device work
runs on the device's current stream, so a page that one call frees may be
written by the next.
"""

from __future__ import annotations

import heapq

import numpy as np
import torch

from . import hga

__all__ = ["OutOfPages", "PageBook", "PagedCache"]

PAGE = 64


class OutOfPages(RuntimeError):
    """Too few free pages; nothing was changed."""


class PageBook:
    """Pages [0, n_pages) are the device's, [n_pages, n_pages + n_cold) the cold
    tier's.  ``table[s, c]`` is the page of chunk c of sequence s (-1: none),
    ``length[s]`` its tokens, ``refs`` how many table entries name a page.

    Methods that change the table note the entries in ``changed`` and return
    the copies to make, (src, dst) pairs in which no dst stands twice or among
    the sources."""

    def __init__(self, n_pages: int, n_seqs: int, max_pages: int, n_cold: int = 0):
        if min(n_pages, n_seqs, max_pages, n_cold) < 0:
            raise ValueError("n_pages, n_seqs, max_pages and n_cold must be >= 0")
        self.n_pages, self.n_cold, self.max_pages = n_pages, n_cold, max_pages
        self.table = np.full((n_seqs, max_pages), -1, np.int32)
        self.length = np.zeros(n_seqs, np.int64)
        self.refs = np.zeros(n_pages + n_cold, np.int64)
        self._free = (list(range(n_pages)), list(range(n_pages, n_pages + n_cold)))  # heaps
        self.changed: set = set()

    # lowest ids first, so that the pages in use stay close together
    def n_free(self, cold: bool = False) -> int:
        return len(self._free[cold])

    def _set(self, s: int, c: int, page: int):
        old = int(self.table[s, c])
        if old == page:
            return
        if page >= 0:
            self.refs[page] += 1
        if old >= 0:
            self.refs[old] -= 1
            if self.refs[old] == 0:
                heapq.heappush(self._free[old >= self.n_pages], old)
        self.table[s, c] = page
        self.changed.add((s, c))

    def _seq(self, s) -> int:
        if not 0 <= int(s) < len(self.length):
            raise ValueError(f"sequence {s} is outside [0, {len(self.length)})")
        return int(s)

    def append(self, seqs, counts):
        """Room for counts[i] more tokens of sequence seqs[i]; raises OutOfPages
        before anything changes."""
        seqs = np.asarray(seqs, np.int64).reshape(-1)
        counts = np.asarray(counts, np.int64).reshape(-1)
        if len(seqs) != len(counts) or (counts < 0).any():
            raise ValueError("append: a count >= 0 for every sequence")
        if len(seqs) and (seqs.min() < 0 or seqs.max() >= len(self.length)):
            raise ValueError(f"append: sequences outside [0, {len(self.length)})")
        if len(np.unique(seqs)) != len(seqs):
            raise ValueError("append: a sequence stands twice")
        now = self.length[seqs]
        have, need = -(-now // PAGE), -(-(now + counts) // PAGE)
        if (need > self.max_pages).any():
            raise ValueError(f"append: more than {self.max_pages} pages a sequence")
        # the last page, if not full, is written too: by this sequence alone, on the device
        last = self.table[seqs, np.maximum(now // PAGE, 0).clip(max=max(self.max_pages - 1, 0))] \
            if self.max_pages else np.full(len(seqs), -1)
        partial = (now % PAGE > 0) & (counts > 0)
        if (partial & (last < 0)).any():
            raise ValueError("append: a sequence's last page is absent")
        # of a call's sequences that share a last page one may keep it, if no other shares it
        uses: dict = {}
        for p in last[partial].tolist():
            uses[p] = uses.get(p, 0) + 1
        copies = sum(n if p >= self.n_pages else min(n, int(self.refs[p]) - 1)
                     for p, n in uses.items())
        if int((need - have).sum()) + copies > self.n_free():
            raise OutOfPages(f"{int((need - have).sum()) + copies} pages wanted, "
                             f"{self.n_free()} free")
        moves = []
        for i in np.nonzero((need > have) | partial)[0].tolist():
            s = int(seqs[i])
            if partial[i] and (self.refs[last[i]] > 1 or last[i] >= self.n_pages):
                page = heapq.heappop(self._free[0])
                moves.append((int(last[i]), page))
                self._set(s, int(now[i]) // PAGE, page)
            for c in range(int(have[i]), int(need[i])):
                self._set(s, c, heapq.heappop(self._free[0]))
        self.length[seqs] += counts
        return moves

    def truncate(self, s: int, length: int):
        """Drop the tokens of sequence s from position `length` on."""
        s = self._seq(s)
        if not 0 <= length <= self.length[s]:
            raise ValueError(f"truncate: {length} is outside [0, {int(self.length[s])}]")
        if length % PAGE and self.table[s, length // PAGE] < 0:
            raise ValueError("truncate: the new last page is absent")
        for c in range(-(-length // PAGE), -(-int(self.length[s]) // PAGE)):
            self._set(s, c, -1)
        self.length[s] = length

    def release(self, s: int):
        """Free a sequence: its pages, but those that others share."""
        s = self._seq(s)
        for c in range(-(-int(self.length[s]) // PAGE)):
            self._set(s, c, -1)
        self.length[s] = 0

    def fork(self, src: int, dst: int):
        """Sequence dst becomes src, sharing its pages."""
        src, dst = self._seq(src), self._seq(dst)
        if src == dst:
            return
        self.release(dst)
        for c in range(-(-int(self.length[src]) // PAGE)):
            self._set(dst, c, int(self.table[src, c]))
        self.length[dst] = self.length[src]

    def _full(self, s: int, begin: int, end: int):
        if not 0 <= begin <= end <= self.length[s] // PAGE:
            raise ValueError(f"chunks [{begin}, {end}) are not full ones of sequence {s}")

    def drop(self, s: int, begin: int, end: int):
        """Full chunks [begin, end) of sequence s become absent: not seen, not
        routed to (a window that has moved on)."""
        s = self._seq(s)
        self._full(s, begin, end)
        for c in range(begin, end):
            self._set(s, c, -1)

    def move(self, s: int, begin: int, end: int, cold: bool):
        """The pages of full chunks [begin, end) of sequence s go to the cold
        tier, or back, for every sequence that shares them."""
        s = self._seq(s)
        self._full(s, begin, end)
        pages = {int(p) for p in self.table[s, begin:end] if p >= 0 and (p >= self.n_pages) != cold}
        if len(pages) > self.n_free(cold):
            raise OutOfPages(f"{len(pages)} pages wanted, {self.n_free(cold)} free")
        return self._replace({p: heapq.heappop(self._free[cold]) for p in sorted(pages)})

    def compact(self):
        """The device's pages in use become [0, how many they are)."""
        used = np.nonzero(self.refs[:self.n_pages])[0]
        n = len(used)
        holes = [p for p in range(n) if self.refs[p] == 0]
        far = [int(p) for p in used if p >= n]
        self._free[0][:] = [p for p in self._free[0] if p >= n]
        heapq.heapify(self._free[0])
        return self._replace(dict(zip(far, holes)))

    def _replace(self, by: dict):
        if by:
            old = np.fromiter(by, np.int32)
            for s, c in zip(*np.nonzero(np.isin(self.table, old))):
                self._set(int(s), int(c), by[int(self.table[s, c])])
        return list(by.items())


class PagedCache:
    """A pool of pages and the sequences in it.

    ``append`` gives the batch of the next tokens, which ``hga_cache_append``
    then stores layer by layer; ``page_table`` (int32 [n_seqs, max_pages], on
    the GPU) is updated in place."""

    def __init__(self, plan: hga.Plan, n_pages: int, n_seqs: int, max_pages: int, n_layers: int = 1,
                 n_cold: int = 0, device="cuda"):
        self.plan = plan
        self.book = PageBook(n_pages, n_seqs, max_pages, n_cold)
        self.pool = hga.Pool(plan, n_pages, n_layers, n_cold, device)
        self.page_table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32,
                                     device=self.pool.device)

    def length(self, s: int) -> int:
        return int(self.book.length[s])

    def _upload(self, x) -> torch.Tensor:
        # pinned memory goes back to its allocator only once the copy has run
        t = torch.from_numpy(np.ascontiguousarray(x)).pin_memory()
        return t.to(self.pool.device, non_blocking=True)

    def _apply(self, moves):
        # the calls ask for the pool's device to be the current one, and the book has changed already
        with torch.cuda.device(self.pool.index):
            self._write(moves)

    def _write(self, moves):
        if moves:
            m = self._upload(np.asarray(moves, np.int32).T)
            hga.hga_copy_pages(self.plan, self.pool, m[0], m[1])
        if self.book.changed:
            at = np.array(sorted(self.book.changed), np.int64)
            self.book.changed.clear()
            new = self.book.table[at[:, 0], at[:, 1]].astype(np.int64)
            up = self._upload(np.stack((at[:, 0] * self.page_table.shape[1] + at[:, 1], new)))
            self.page_table.view(-1).index_copy_(0, up[0], up[1].int())

    def append(self, seqs, counts) -> hga.TokenBatch:
        """The next counts[i] tokens of sequence seqs[i], in order.  The batch's
        tensors are new ones: for a captured step copy its tok_seq and tok_pos
        into those of the batch it was captured with."""
        seqs, counts = np.asarray(seqs, np.int64).reshape(-1), np.asarray(counts, np.int64).reshape(-1)
        moves = self.book.append(seqs, counts)
        self._apply(moves)
        n = int(counts.sum())
        tok = np.empty((2, n), np.int32)
        tok[0] = np.repeat(seqs, counts)
        start = self.book.length[seqs] - counts
        tok[1] = np.arange(n) - np.repeat(np.cumsum(counts) - counts, counts) + np.repeat(start, counts)
        tok = self._upload(tok)
        return hga.TokenBatch(tok[0], tok[1], self.page_table)

    def truncate(self, s: int, length: int):
        """As PageBook.truncate; so the methods that follow."""
        self.book.truncate(s, length)
        self._apply(None)

    def release(self, s: int):
        self.book.release(s)
        self._apply(None)

    def fork(self, src: int, dst: int):
        self.book.fork(src, dst)
        self._apply(None)

    def drop(self, s: int, begin: int, end: int):
        self.book.drop(s, begin, end)
        self._apply(None)

    def to_cold(self, s: int, begin: int, end: int) -> int:
        """Full chunks [begin, end) into host memory; how many pages moved."""
        moves = self.book.move(s, begin, end, True)
        self._apply(moves)
        return len(moves)

    def to_device(self, s: int, begin: int, end: int) -> int:
        moves = self.book.move(s, begin, end, False)
        self._apply(moves)
        return len(moves)

    def compact(self) -> int:
        moves = self.book.compact()
        self._apply(moves)
        return len(moves)
