"""Which sequences of a PageBook begin with the same pages, and evictions from
it, on the host; the checks of hga_attend_shared, hga_weigh_pages and
hga_choose_evictions, compiled for the CPU."""

from __future__ import annotations

import itertools
import os
import subprocess

import numpy as np
import pytest

from paper_2606_30709_amd import build
from paper_2606_30709_amd.pages import PAGE, PageBook

HERE = os.path.dirname(os.path.abspath(__file__))


def test_bounds_and_refusals(tmp_path):
    exe = str(tmp_path / "prefixes_check")
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-w",
                    "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "prefixes_check.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def _alike(book, members):
    n = min(int(book.length[s]) // PAGE for s in members)
    rows = book.table[list(members), :n]
    differ = np.nonzero((rows != rows[0]).any(0))[0]
    return int(differ[0]) if len(differ) else n


def _saved(book, groups):
    assert len({s for m, _ in groups for s in m}) == sum(len(m) for m, _ in groups)
    for members, pages in groups:
        assert len(members) >= 2 and 0 < pages <= _alike(book, members)
    return sum((len(m) - 1) * p for m, p in groups)


def _most(book, seqs):
    """The most pages that any partition saves."""
    if not seqs:
        return 0
    first, rest = seqs[0], seqs[1:]
    best = _most(book, rest)
    for n in range(1, len(rest) + 1):
        for with_ in itertools.combinations(rest, n):
            best = max(best, n * _alike(book, (first, *with_)) + _most(book, [s for s in rest if s not in with_]))
    return best


def test_groups_of_forks():
    book = PageBook(100, 6, 12)
    assert book.groups([]) == [] and book.groups([0, 3]) == []
    book.append([0], [PAGE * 4 + 10])
    for s in (1, 2):
        book.fork(0, s)
    assert book.groups([2, 0, 1]) == [([2, 0, 1], 4)]
    assert book.groups([0]) == [] and book.groups([0, 5]) == []
    book.append([1], [PAGE * 3])
    book.fork(1, 3)
    # 0 and 2 share four pages, 1 and 3 seven: together 12 saved, apart 4 + 7
    assert book.groups([0, 1, 2, 3]) == [([0, 1, 2, 3], 4)]
    book.release(2)
    # three sequences over four pages save 8, two over seven 7
    assert book.groups([0, 1, 3]) == [([0, 1, 3], 4)]
    book.truncate(0, PAGE * 2)
    assert book.groups([0, 1, 3]) == [([1, 3], 7)]
    with pytest.raises(ValueError):
        book.groups([0, 0])
    with pytest.raises(ValueError):
        book.groups([6])


def test_groups_save_the_most():
    rng = np.random.default_rng(0)
    for _ in range(60):
        n = int(rng.integers(2, 7))
        book = PageBook(400, n, 30)
        book.append([0], [int(rng.integers(1, 20)) * 40])
        for s in range(1, n):
            if rng.random() < 0.8:
                src = int(rng.integers(0, s))
                book.fork(src, s)
                book.truncate(s, int(rng.integers(0, book.length[s] + 1)))
            book.append([s], [int(rng.integers(0, 300))])
        if rng.random() < 0.3:
            s = int(rng.integers(0, n))
            full = int(book.length[s]) // PAGE
            if full > 1:
                book.drop(s, 0, 1)
        seqs = rng.permutation(n).tolist()
        assert _saved(book, book.groups(seqs)) == _most(book, seqs)


def test_groups_of_a_long_chain_of_forks():
    n = 3000
    book = PageBook(2 * n + 10, n, n + 1)
    for s in range(n):
        if s:
            book.fork(s - 1, s)
            if s > 40:   # (few pages each, a chain all the same)
                book.truncate(s, PAGE * 40)
        book.append([s], [PAGE])
    assert _saved(book, book.groups(range(n))) >= 40 * (n - 41)


def test_evicted_pages():
    book = PageBook(20, 2, 8)
    book.append([0], [PAGE * 5 + 1])
    book.fork(0, 1)
    table = book.table.copy()
    with pytest.raises(ValueError):
        book.evict(0, [1, 5])          # the last is not full: nothing is done
    assert np.array_equal(table, book.table)
    book.evict(0, [1, 3])
    assert (book.table[0, :6] >= 0).tolist() == [True, False, True, False, True, True]
    assert np.array_equal(table[1], book.table[1]) and book.n_free() == 14
    book.evict(1, [1])
    assert book.n_free() == 15 and book.groups([0, 1]) == [([0, 1], 3)]
