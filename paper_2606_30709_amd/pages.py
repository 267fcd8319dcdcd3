"""Sequences in the pages of a cache: allocation, sharing, copying, moving.

``PageBook`` is the host's part: which page holds which chunk of which
sequence, how many sequences share a page and which begin with the same pages,
which pages are free.  It touches no
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

    def evict(self, s: int, chunks):
        """The given full chunks of sequence s become absent, as by drop."""
        s = self._seq(s)
        chunks = [int(c) for c in chunks]
        for c in chunks:
            self._full(s, c, c + 1)
        for c in chunks:
            self._set(s, c, -1)

    def groups(self, seqs):
        """Which of the given sequences begin with the same pages, as (sequences,
        pages) of each group of two or more, in the order given: grouped so that the most pages are
        read once instead of by each.  Only pages full in all of a group count (so
        that no later append gives one of them a page of its own); absent ones of
        all count as the same."""
        seqs = [self._seq(s) for s in seqs]
        if len(set(seqs)) != len(seqs):
            raise ValueError("groups: a sequence stands twice")
        full = {s: int(self.length[s]) // PAGE for s in seqs}
        # Nodes: sequences that are alike up to `shared`, and then go apart.  If a group is formed at a node, its
        # sequences that no deeper group takes save `shared` pages each, but for one of them.  above: what a sequence
        # saves in a group of one of the nodes above (0: in none).
        nodes, todo = [], [(seqs, 0, -1, np.zeros(1, np.int64))]
        while todo:
            members, at, parent, above = todo.pop()
            rows = self.table[members, at:min((full[s] for s in members), default=0)]
            differ = np.nonzero((rows != rows[:1]).any(0))[0]
            shared = at + (int(differ[0]) if len(differ) else rows.shape[1])
            parts: dict = {}
            for s in members:
                parts.setdefault(int(self.table[s, shared]) if full[s] > shared else ~s - 1, []).append(s)
            own = [p[0] for p in parts.values() if len(p) == 1]
            below = np.append(above, shared)
            todo += [(p, shared, len(nodes), below) for p in parts.values() if len(p) > 1]
            nodes.append([own, shared, parent, above, len(own) * below, None])
        for node in reversed(nodes):    # the pages saved, with a group here and without
            _, shared, parent, _, saved, _ = node
            node[5] = saved[-1] - shared > saved[:-1]
            if parent >= 0:
                nodes[parent][4] = nodes[parent][4] + np.maximum(saved[-1] - shared, saved[:-1])
        result, taken = [], []          # the group that a node's sequences are in, and its place in `above`
        for own, shared, parent, above, _, better in nodes:
            group, place = taken[parent] if parent >= 0 else (None, 0)
            if better[place]:
                group, place = ([], shared), len(above)
                result.append(group)
            taken.append((group, place))
            if group is not None:
                group[0].extend(own)
        rank = {s: i for i, s in enumerate(seqs)}
        return sorted(((sorted(members, key=rank.get), shared) for members, shared in result),
                      key=lambda g: rank[g[0][0]])

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
    the GPU) is updated in place, and so is what ``page_weights`` gave."""

    _weights = None  # what page_weights gave

    def __init__(self, plan: hga.Plan, n_pages: int, n_seqs: int, max_pages: int, n_layers: int = 1,
                 n_cold: int = 0, device="cuda"):
        self.plan = plan
        self.book = PageBook(n_pages, n_seqs, max_pages, n_cold)
        self.pool = hga.Pool(plan, n_pages, n_layers, n_cold, device)
        self.page_table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32,
                                     device=self.pool.device)

    def page_weights(self) -> torch.Tensor:
        """The cache's own attention weights of pages, fp32 [n_layers, n_seqs,
        n_kv_heads, max_pages], zeros before the first call, the same tensor in
        every call: ``TokenPipeline.step`` adds a layer's to it, ``evict`` goes by
        its sum over layers, or one layer.  They go with their sequences: ``fork``
        copies them, ``release`` clears them, ``truncate`` those of the chunks it
        drops (a chunk that it cuts keeps what the chunk had).  In a tensor of the
        caller's own that is left to the caller: without it a row's next sequence
        goes on from the last one's weights."""
        if self._weights is None:
            if torch.cuda.is_current_stream_capturing():
                raise hga.HgaError(-1, "HGA_EINVAL: the page weights of a captured step have to be there before it")
            p = self.plan.params
            self._weights = torch.zeros(self.pool.n_layers, len(self.book.length), p.n_kv_heads, self.book.max_pages,
                                        dtype=torch.float32, device=self.pool.device)
        return self._weights

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

    def prefixes(self, batch: hga.TokenBatch, seqs, counts) -> hga.Prefixes | None:
        """What the batch that ``append(seqs, counts)`` gave shares, for
        hga_attend_shared (None: nothing).  It stays valid for batches of the same
        counts while their sequences only grow or move (``to_cold``, ``to_device``,
        ``compact``); a sequence of it that is cut, dropped from, evicted from,
        forked over or released needs another one.  Its hints are those of the
        lengths now."""
        seqs, counts = np.asarray(seqs, np.int64).reshape(-1), np.asarray(counts, np.int64).reshape(-1)
        if int(counts.sum()) != batch.n_tokens:
            raise ValueError(f"prefixes: {int(counts.sum())} tokens, the batch has {batch.n_tokens}")
        some = counts > 0
        groups = self.book.groups(seqs[some].tolist())
        if not groups:
            return None
        start = dict(zip(seqs.tolist(), (np.cumsum(counts) - counts).tolist()))
        n = dict(zip(seqs.tolist(), counts.tolist()))
        pages = {s: p for members, p in groups for s in members}
        slots = [t for members, _ in groups for s in members for t in range(start[s], start[s] + n[s])]
        alone = [t for s in seqs[some].tolist() if s not in pages for t in range(start[s], start[s] + n[s])]
        begin = np.cumsum([0] + [sum(n[s] for s in members) for members, _ in groups])
        own = max(-(-int(self.book.length[s]) // PAGE) - pages.get(s, 0) for s in seqs[some].tolist())
        up = self._upload(np.concatenate((slots, alone, begin, [p for _, p in groups])).astype(np.int32))
        # (the calls ask for alignment to four bytes alone)
        order, begin, shared = up.split((batch.n_tokens, len(groups) + 1, len(groups)))
        return hga.Prefixes(order, begin, shared, max(p for _, p in groups), max(own, 1))

    def evict(self, weights: torch.Tensor, budget, together: bool = False) -> list:
        """Drop of each sequence s the pages above budget[s] (an int: of every one;
        one below 0 counts as 0) that hga_choose_evictions names by ``weights``
        (fp32 [n_seqs, n_kv_heads, max_pages]: those of one layer, or a sum over
        them, see ``page_weights``); the chunks dropped, a list for each sequence.
        Waits for the device; the weights are not changed (an absent page gets
        nothing more).

        A page that sequences share is free only when all of them have dropped it,
        and those that drop different pages begin with fewer in common
        (``prefixes``).  Each sequence by itself chooses by its own weights;
        together: a page counts in all of its sequences by what it got of all of
        them, so that forks drop the same pages of their prompt, one with a smaller
        budget (or a shorter window) those and the next ones."""
        book = self.book
        n_seqs = len(book.length)
        want = np.broadcast_to(np.asarray(budget, np.int64), (n_seqs,)).clip(0, 2 ** 31 - 1)
        here = (book.table >= 0).sum(1)
        most = int((here - want).clip(0).max(initial=0))
        if most == 0:
            return [[] for _ in range(n_seqs)]
        dev = self.pool.device
        with torch.cuda.device(self.pool.index):
            state = self._upload(np.stack((book.length, want)).astype(np.int32))
            out = torch.empty(n_seqs, most, dtype=torch.int32, device=dev)
            if together:
                weights = self._of_sharers(weights)
            nbytes = hga.hga_choose_evictions_workspace(self.plan, self.page_table)
            ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
            hga.hga_choose_evictions(self.plan, self.page_table, book.n_pages + book.n_cold, state[0], weights,
                                     state[1], out, workspace=ws)
            chosen = [[c for c in row if c >= 0] for row in out.tolist()]
        for s, chunks in enumerate(chosen):
            book.evict(s, chunks)
        self._apply(None)
        return chosen

    def _of_sharers(self, weights: torch.Tensor) -> torch.Tensor:
        """weights, a page's that sequences share the sum of theirs: in 64 bits, a
        sequence at a time, so that it is the same in each of them and every time."""
        book, kv = self.book, self.plan.params.n_kv_heads
        hga._expect(weights, "weights", torch.float32, (*book.table.shape[:1], kv, book.max_pages), self.pool.device)
        rows, chunks = np.nonzero((book.table >= 0) & (book.refs[book.table] > 1))
        if not len(rows):
            return weights
        at = self._upload(np.stack((chunks, book.table[rows, chunks])).astype(np.int64))
        counts = np.bincount(rows, minlength=len(book.length)).tolist()
        parts = [(s, *x) for s, x in enumerate(zip(*(y.split(counts) for y in at))) if counts[s]]
        total = torch.zeros(kv, book.n_pages + book.n_cold, dtype=torch.float64, device=weights.device)
        for s, c, page in parts:     # (no page stands twice in a row)
            total[:, page] += weights[s][:, c].double()
        weights = weights.clone()
        for s, c, page in parts:
            weights[s].index_copy_(1, c, total[:, page].float())
        return weights

    def truncate(self, s: int, length: int):
        """As PageBook.truncate; so the methods that follow."""
        self.book.truncate(s, length)
        self._apply(None)
        self._forget(s, -(-length // PAGE))

    def release(self, s: int):
        self.book.release(s)
        self._apply(None)
        self._forget(s, 0)

    def fork(self, src: int, dst: int):
        self.book.fork(src, dst)
        self._apply(None)
        if self._weights is not None and src != dst:
            with torch.cuda.device(self.pool.index):
                self._weights[:, dst] = self._weights[:, src]

    def _forget(self, s: int, begin: int):
        """The page weights of sequence s from chunk `begin` on become zeros."""
        if self._weights is not None:
            with torch.cuda.device(self.pool.index):
                self._weights[:, s, :, begin:].zero_()

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
