"""The page weights that a PagedCache keeps: they go with their sequences through
forks, cuts and releases, and evictions by them are those of the sequence's own
history."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import prefix_util as P
from tokens_util import PAGE, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


class _Cache:
    def __init__(self, hga, n_seqs=4, layers=2, routed=False):
        from paper_2606_30709_amd.pages import PagedCache
        from paper_2606_30709_amd.pipeline import TokenPipeline
        self.plan = hga.Plan(batch=1, n_q_heads=4, n_kv_heads=2, head_dim=64, keep_first=1, keep_last=1, topk_chunks=3,
                             topk_groups=4)
        self.cache = PagedCache(self.plan, 120, n_seqs, 20, n_layers=layers)
        self.pipe, self.layers = TokenPipeline(self.cache, routed), layers
        self.g = torch.Generator().manual_seed(3)

    def rand(self, *s):
        return torch.randn(*s, generator=self.g).bfloat16().cuda()

    def serve(self, seqs, counts):
        batch = self.cache.append(seqs, counts)
        for layer in range(self.layers):
            self.pipe.step(layer, batch, self.rand(batch.n_tokens, 4, 64), self.rand(batch.n_tokens, 2, 64),
                           self.rand(batch.n_tokens, 2, 64), weights=self.cache.page_weights()[layer])


def test_weights_go_with_their_sequences(hga):
    t = _Cache(hga)
    cache = t.cache
    w = cache.page_weights()
    assert w.shape == (2, 4, 2, 20) and w.dtype == torch.float32 and not w.any()
    t.serve([0, 1], [PAGE * 9 + 5, PAGE * 12])
    before = w.clone()
    assert (before[:, 0, :, :10] > 0).all() and not before[:, 0, :, 10:].any() and not before[:, 2:].any()
    cache.fork(0, 2)
    cache.fork(1, 1)
    assert torch.equal(w[:, 2], before[:, 0]) and torch.equal(w[:, :2], before[:, :2]) and not w[:, 3].any()
    cache.fork(2, 1)             # a row that held another sequence
    assert torch.equal(w[:, 1], before[:, 0])
    cache.truncate(2, PAGE * 4)
    assert torch.equal(w[:, 2, :, :4], before[:, 0, :, :4]) and not w[:, 2, :, 4:].any()
    cache.truncate(1, PAGE * 4 + 1)     # cuts chunk 4, which keeps what it had
    assert torch.equal(w[:, 1, :, :5], before[:, 0, :, :5]) and not w[:, 1, :, 5:].any()
    cache.drop(1, 1, 3)
    cache.compact()
    assert torch.equal(w[:, 0], before[:, 0])
    cache.release(0)
    assert not w[:, 0].any() and w[:, 1].any()
    cache.truncate(1, 0)
    assert not w[:, 1].any()
    for bad in (lambda: cache.truncate(2, PAGE * 5), lambda: cache.release(9), lambda: cache.fork(9, 2)):
        kept = w.clone()
        with pytest.raises(ValueError):
            bad()
        assert torch.equal(w, kept)
    assert cache.page_weights() is w


def test_a_reused_row_is_evicted_by_its_own_history(hga):
    """A sequence in a row that held another, and a fork, against the same ones in
    a cache of their own."""
    used, fresh = _Cache(hga), _Cache(hga)
    used.serve([0, 1], [PAGE * 18, PAGE * 15])
    used.cache.release(0)
    used.cache.truncate(1, 0)
    used.g.manual_seed(9), fresh.g.manual_seed(9)
    for t in (used, fresh):
        t.serve([0], [PAGE * 16 + 9])
        t.serve([1], [PAGE * 8 + 1])
        t.cache.fork(0, 3)
        t.serve([3, 0], [1, 1])
    for x in (0, 1, 3):
        assert torch.equal(used.cache.page_weights()[:, x], fresh.cache.page_weights()[:, x])
    total = [t.cache.page_weights().sum(0) for t in (used, fresh)]
    gone = [t.cache.evict(w, [10, 6, 20, 5]) for t, w in zip((used, fresh), total)]
    assert gone[0] == gone[1] and [len(x) for x in gone[0]] == [7, 3, 0, 12]
    book = used.cache.book
    length = np.array([PAGE * 16 + 10, PAGE * 8 + 1, 0, PAGE * 16 + 10])
    table = np.full((4, 20), -1, np.int32)
    for s, n in enumerate(length):
        table[s, :-(-n // PAGE)] = 1
    want = P.choose(table, 2, length, f64(total[0]).astype(np.float32), [10, 6, 20, 5], 12, 1, 1)
    assert gone[0] == [[c for c in row if c >= 0] for row in want.tolist()]
    assert book.n_free() == fresh.cache.book.n_free()


def test_weights_with_a_captured_step(hga):
    """Replays add to the cache's tensor, also behind a release."""
    t, other = _Cache(hga, layers=1), _Cache(hga, layers=1)
    with pytest.raises(hga.HgaError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            t.cache.page_weights()
    for x in (t, other):
        x.serve([0, 1], [PAGE * 3, PAGE * 5 + 7])
        x.cache.fork(1, 2)
    seqs, ones = [0, 1, 2], [1, 1, 1]
    batch = t.cache.append(seqs, ones)
    q, k, v = t.rand(3, 4, 64), t.rand(3, 2, 64), t.rand(3, 2, 64)
    w = t.cache.page_weights()
    t.pipe.step(0, batch, q, k, v, weights=w[0])
    other.pipe.step(0, other.cache.append(seqs, ones), q, k, v, weights=other.cache.page_weights()[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.pipe.step(0, batch, q, k, v, weights=w[0])
    for i in range(6):
        for x in (q, k, v):
            x.copy_(t.rand(*x.shape))
        if i == 3:
            for x in (t, other):
                x.cache.release(0)
                x.cache.fork(2, 0)
        b = t.cache.append(seqs, ones)
        batch.tok_seq.copy_(b.tok_seq)
        batch.tok_pos.copy_(b.tok_pos)
        graph.replay()
        other.pipe.step(0, other.cache.append(seqs, ones), q, k, v, weights=other.cache.page_weights()[0])
        assert torch.equal(w, other.cache.page_weights()) and w[0, :3].any()
