"""The page bookkeeping against a model that holds every token of every sequence
by itself: what a page holds is what its sequences' tokens are, whatever was
appended, forked, dropped, moved and freed before."""

from __future__ import annotations

import random

import numpy as np
import pytest

from paper_2606_30709_amd.pages import PAGE, OutOfPages, PageBook


class _Model:
    """Rows of pages as the device would hold them, and sequences as lists."""

    def __init__(self, book):
        self.book, self.next = book, 0
        self.rows = np.full((book.n_pages + book.n_cold, PAGE), -1)
        self.seqs = [[] for _ in book.length]
        self.gone = [set() for _ in book.length]

    def copy(self, moves):
        moves = moves or []
        src, dst = [m[0] for m in moves], [m[1] for m in moves]
        assert len(set(dst)) == len(dst) and not set(src) & set(dst)
        for s, d in moves:
            self.rows[d] = self.rows[s]

    def append(self, seqs, counts):
        self.copy(self.book.append(seqs, counts))
        wrote = set()
        for s, n in zip(seqs, counts):
            for _ in range(n):
                p = len(self.seqs[s])
                page = self.book.table[s, p // PAGE]
                assert (page, p % PAGE) not in wrote and page < self.book.n_pages
                wrote.add((page, p % PAGE))
                self.rows[page, p % PAGE] = self.next
                self.seqs[s].append(self.next)
                self.next += 1

    def check(self):
        b = self.book
        refs = np.bincount(b.table[b.table >= 0], minlength=len(b.refs)) if len(b.refs) else b.refs
        assert np.array_equal(refs, b.refs)
        for cold in (False, True):
            lo, hi = (b.n_pages, b.n_pages + b.n_cold) if cold else (0, b.n_pages)
            assert sorted(b._free[cold]) == [p for p in range(lo, hi) if refs[p] == 0]
        for s, toks in enumerate(self.seqs):
            assert b.length[s] == len(toks)
            n = -(-len(toks) // PAGE)
            assert (b.table[s, n:] == -1).all()
            for c in range(n):
                if c in self.gone[s]:
                    assert b.table[s, c] == -1
                else:
                    part = toks[c * PAGE:(c + 1) * PAGE]
                    assert list(self.rows[b.table[s, c], :len(part)]) == part


@pytest.mark.parametrize("seed", range(12))
def test_pages_hold_their_sequences(seed):
    rng = random.Random(seed)
    book = PageBook(rng.randint(4, 40), rng.randint(1, 6), rng.randint(2, 12), rng.randint(0, 9))
    m = _Model(book)
    n = len(book.length)
    for _ in range(300):
        do = rng.choice(["append"] * 4 + ["truncate", "release", "fork", "fork", "drop", "move", "compact"])
        s = rng.randrange(n)
        size = len(m.seqs[s])
        before = (book.table.copy(), book.length.copy(), book.refs.copy())
        try:
            if do == "append":
                seqs = rng.sample(range(n), rng.randint(1, n))
                m.append(seqs, [rng.choice([0, 1, 1, rng.randint(0, 150)]) for _ in seqs])
            elif do == "truncate":
                k = rng.randint(0, size)
                book.truncate(s, k)
                m.seqs[s] = m.seqs[s][:k]
                m.gone[s] = {c for c in m.gone[s] if c * PAGE < k}
            elif do == "release":
                book.release(s)
                m.seqs[s], m.gone[s] = [], set()
            elif do == "fork":
                d = rng.randrange(n)
                book.fork(s, d)
                m.seqs[d], m.gone[d] = list(m.seqs[s]), set(m.gone[s])
            elif do == "drop":
                a = rng.randint(0, size // PAGE)
                e = rng.randint(a, size // PAGE)
                book.drop(s, a, e)
                m.gone[s] |= set(range(a, e))
            elif do == "move":
                a = rng.randint(0, size // PAGE)
                e, cold = rng.randint(a, size // PAGE), rng.random() < 0.6
                m.copy(book.move(s, a, e, cold))
                for c in range(a, e):
                    assert book.table[s, c] == -1 or (book.table[s, c] >= book.n_pages) == cold
            else:
                m.copy(book.compact())
                used = np.nonzero(book.refs[:book.n_pages])[0]
                assert list(used) == list(range(len(used)))
        except (OutOfPages, ValueError):
            # refused before anything changed
            assert all(np.array_equal(x, y) for x, y in zip(before, (book.table, book.length, book.refs)))
        m.check()


def test_bookkeeping_refuses():
    book = PageBook(4, 2, 3, 1)
    for f in (lambda: book.append([0, 0], [1, 1]), lambda: book.append([2], [1]), lambda: book.append([0], [-1]),
              lambda: book.append([0, 1], [1]), lambda: book.append([0], [3 * PAGE + 1]), lambda: book.truncate(0, 1),
              lambda: book.fork(0, 2), lambda: book.release(-1), lambda: book.drop(0, 0, 1),
              lambda: book.move(0, 0, 1, True), lambda: PageBook(-1, 1, 1)):
        with pytest.raises(ValueError):
            f()
    book.append([0], [2 * PAGE + 5])
    with pytest.raises(OutOfPages):
        book.append([1], [PAGE + 1])
    with pytest.raises(OutOfPages):
        book.move(0, 0, 2, True)
    with pytest.raises(ValueError):
        book.drop(0, 0, 3)             # the last one is not full
    book.fork(0, 1)
    # both append to the shared page: one of them keeps it
    moves = book.append([0, 1], [1, 1])
    assert len(moves) == 1 and book.n_free() == 0
    assert PageBook(0, 0, 0).append([], []) == []
    assert sorted(book.changed) == sorted(set(book.changed))
