"""PagedCache.evict: its budgets, and what it frees of pages that sequences share.
On the host the choice is prefix_util's."""

from __future__ import annotations

import contextlib
import types

import numpy as np
import pytest
import torch

import prefix_util as P
from paper_2606_30709_amd import hga, pages
from tokens_util import PAGE


class _Params(types.SimpleNamespace):
    n_kv_heads = 2


@pytest.fixture
def cache(monkeypatch):
    """A cache on the host; lists are no longer than the table is wide."""
    def choose(plan, table, n_ids, seq_len, weights, budget, evicted, workspace=None, stream=None):
        assert evicted.shape[1] <= table.shape[1]
        evicted.copy_(torch.from_numpy(P.choose(table.numpy(), n_ids, seq_len.numpy(), weights.numpy(), budget.numpy(),
                                                evicted.shape[1], 1, 1)))

    monkeypatch.setattr(torch.cuda, "device", lambda index: contextlib.nullcontext())
    monkeypatch.setattr(pages.hga, "hga_choose_evictions", choose)
    monkeypatch.setattr(pages.hga, "hga_choose_evictions_workspace", lambda plan, table: 0)
    monkeypatch.setattr(pages.PagedCache, "_upload", lambda self, x: torch.from_numpy(np.ascontiguousarray(x)))
    c = pages.PagedCache.__new__(pages.PagedCache)
    c.plan, c.book = types.SimpleNamespace(params=_Params()), pages.PageBook(80, 5, 20)
    c.pool = types.SimpleNamespace(index=0, device=torch.device("cpu"))
    c.page_table = torch.full((5, 20), -1, dtype=torch.int32)
    return c


def test_budgets_of_any_size(cache):
    cache.book.append([0, 1], [PAGE * 9 + 1, PAGE * 4])
    cache._apply(None)
    w = torch.rand(5, 2, 20)
    for budget in (-1, -2 ** 31, -2 ** 62):
        # the first page, the window and the last one stay
        assert [len(x) for x in cache.evict(w, [2 ** 62, budget, 0, 0, 0])] == [0, 1, 0, 0, 0]
        cache.book.truncate(1, 0)
        cache.book.append([1], [PAGE * 4])
        cache._apply(None)
    assert cache.evict(w, 10) == [[]] * 5


def _free_and_groups(cache, seqs):
    return cache.book.n_free(), cache.book.groups(seqs)


def test_sequences_by_themselves_drop_pages_of_their_own_choice(cache):
    """What the docstring says of shared pages: none is freed before all have
    dropped it, and the common prefix ends where the first of them has."""
    book = cache.book
    book.append([0], [PAGE * 16])
    for s in (1, 2, 3):
        book.fork(0, s)
    cache._apply(None)
    w = torch.full((5, 2, 20), 9.0)
    for s in range(4):
        w[s, :, 2 + 3 * s:5 + 3 * s] = 0.0
    assert cache.evict(w, 13) == [[2, 3, 4], [5, 6, 7], [8, 9, 10], [11, 12, 13], []]
    free, groups = _free_and_groups(cache, range(4))
    assert free == 80 - 16 and max(p for _, p in groups) <= 8
    assert np.array_equal(cache.page_table.numpy(), book.table)


def test_forks_that_evict_together_free_pages_and_stay_a_group(cache):
    book = cache.book
    book.append([0], [PAGE * 16])
    for s in (1, 2, 3):
        book.fork(0, s)
    book.append([4, 3], [PAGE * 8, 2 * PAGE])
    cache._apply(None)
    rng = np.random.default_rng(1)
    w = torch.from_numpy(np.exp(3 * rng.standard_normal((5, 2, 20))).astype(np.float32))
    kept = w.clone()
    free = book.n_free()
    want = kept.double()[:4, :, :16].sum(0)           # what a page of the prompt got of all
    gone = cache.evict(w, [12, 12, 12, 14, 8], together=True)
    assert torch.equal(w, kept)
    order = (1 + np.argsort(want.sum(0)[1:14].numpy(), kind="stable")).tolist()
    assert gone[:3] == [sorted(order[:4])] * 3 and gone[4] == []
    # a page of sequence 3's own counts by itself: it goes first if it got less than the prompt's
    assert set(gone[3]) - {16} <= set(order[:4]) and len(gone[3]) == 4
    common = set(gone[3]) & set(order[:4])
    assert book.n_free() == free + len(common) + (16 in gone[3])
    shared = 16 if len(common) == 4 else min(set(order[:4]) - common)
    assert (list(range(4)), shared) in book.groups(range(5)) or ([0, 1, 2], 16) in book.groups(range(5))
    assert np.array_equal(cache.page_table.numpy(), book.table)
    # smaller budgets drop the same pages and the next ones
    more = cache.evict(w, [10, 9, 10, 20, 20], together=True)
    assert more[0] == more[2] and set(more[0]) <= set(more[1])
    # nothing shared: as each by itself
    for s in (1, 2, 3):
        cache.book.release(s)
    alone = P.choose(book.table, 80, book.length, w.numpy(), [5] * 5, 16, 1, 1)
    assert cache.evict(w, 5, together=True) == [[c for c in row if c >= 0] for row in alone.tolist()]
    with pytest.raises(hga.HgaError):
        cache.evict(w[:, :1], 1, together=True)


@pytest.mark.gpu
def test_samples_evicted_together():
    """On the device: prompts' pages are freed, the samples go on as one group, and
    the choice is that of the definition over the summed weights, every time."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    plan = hga.Plan(batch=1, n_q_heads=6, n_kv_heads=3, head_dim=64, keep_first=1, keep_last=2, topk_chunks=3,
                    topk_groups=4)
    rng = np.random.default_rng(2)
    w = torch.from_numpy(np.exp(3 * rng.standard_normal((9, 3, 60))).astype(np.float32)).cuda()
    w[:, :, 20:24] = 0                                # ties
    before = None
    for _ in range(3):
        cache = pages.PagedCache(plan, 140, 9, 60, n_cold=20)
        cache.append([0, 8], [PAGE * 40 + 3, PAGE * 30])
        for s in range(1, 8):
            cache.fork(0, s)
        cache.append(range(8), [1] * 8)
        cache.to_cold(3, 5, 15)
        free = cache.book.n_free(), cache.book.n_free(True)
        book, kept = cache.book, w.clone()
        total = w.double().cpu().numpy()
        total[:8, :, :40] = total[:8, :, :40].sum(0)
        want = P.choose(book.table, 160, book.length, total.astype(np.float32), [30] * 9, 60, 1, 2)
        gone = cache.evict(w, 30, together=True)
        assert gone == [[c for c in row if c >= 0] for row in want.tolist()] and torch.equal(w, kept)
        assert gone[8] == [] and len(gone[0]) == 11 and all(g == gone[0] for g in gone[:8])
        assert sum(book.n_free(x) for x in (False, True)) == sum(free) + 11
        assert book.groups(range(9)) == [(list(range(8)), 40)]
        assert np.array_equal(cache.page_table.cpu().numpy(), book.table)
        assert before in (None, gone)
        before = gone
