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
