"""PagedCache's device work, on the host: the pool's device is made the current
one for it, since a copy that is refused would find the book changed already."""

from __future__ import annotations

import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2606_30709_amd import hga, pages


@pytest.fixture
def cache(monkeypatch):
    """A cache on device 0 while device 1 is current; copies noted."""
    state = types.SimpleNamespace(device=1, copies=[])

    @contextlib.contextmanager
    def device(index):
        before, state.device = state.device, index
        try:
            yield
        finally:
            state.device = before

    def copy(plan, pool, src, dst, stream=None):
        hga._on(pool, 0)  # refuses another current device
        state.copies += list(zip(src.tolist(), dst.tolist()))

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: state.device)
    monkeypatch.setattr(pages.hga, "hga_copy_pages", copy)
    monkeypatch.setattr(pages.hga, "TokenBatch", lambda seq, pos, table: (seq, pos, table))
    monkeypatch.setattr(pages.PagedCache, "_upload", lambda self, x: torch.from_numpy(np.ascontiguousarray(x)))
    c = pages.PagedCache.__new__(pages.PagedCache)
    c.plan, c.book = None, pages.PageBook(8, 3, 4, 4)
    c.pool = types.SimpleNamespace(index=0, device=torch.device("cpu"))
    c.page_table = torch.full((3, 4), -1, dtype=torch.int32)
    c.state = state
    return c


def test_pages_move_while_another_device_is_current(cache):
    cache.append([0], [130])
    cache.fork(0, 1)
    cache.append([1], [1])                # a copy of the shared last page
    assert len(cache.state.copies) == 1 and cache.state.device == 1
    cache.to_cold(0, 0, 2)
    cache.compact()
    cache.to_device(0, 0, 1)
    cache.release(1)
    assert cache.state.device == 1
    assert np.array_equal(cache.page_table.numpy(), cache.book.table)
