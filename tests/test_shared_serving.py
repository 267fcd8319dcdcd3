"""Samples of one prompt served over shared pages, their pages weighed and
evicted, and served on: PagedCache, TokenPipeline and the operators together,
against 64-bit definitions over what the pages hold."""

from __future__ import annotations

import types

import numpy as np
import pytest
import torch

import prefix_util as P
import tokens_util as U
from tokens_util import f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


class _Served:
    def __init__(self, hga, dtype, d, kv, ratio, routed, layers=2):
        from paper_2606_30709_amd.pages import PagedCache
        from paper_2606_30709_amd.pipeline import TokenPipeline
        self.hga, self.dtype, self.d, self.kv, self.hq, self.layers = hga, dtype, d, kv, kv * ratio, layers
        self.plan = hga.Plan(batch=1, n_q_heads=self.hq, n_kv_heads=kv, head_dim=d, keep_first=1, keep_last=2,
                             topk_chunks=3, topk_groups=4, dtype=hga.F32 if dtype == "f32" else hga.BF16)
        self.cache = PagedCache(self.plan, 120, 6, 24, n_layers=layers, n_cold=5)
        self.pipe, self.routed = TokenPipeline(self.cache, routed), routed
        self.weights = torch.zeros(layers, 6, kv, 24, device="cuda")
        self.want, self.tol = np.zeros((layers, 6, kv, 24)), np.zeros((layers, 6, kv, 24))
        self.rng = np.random.default_rng(5)

    def rand(self, *s):
        return torch.from_numpy(self.rng.standard_normal(s).astype(np.float32)).to(U.DT[self.dtype]).cuda()

    def serve(self, seqs, counts, share=True):
        batch = self.cache.append(seqs, counts)
        px = self.cache.prefixes(batch, seqs, counts) if share and not self.routed else None
        T, n_ids = batch.n_tokens, self.cache.book.n_pages + self.cache.book.n_cold
        seq, pos = (x.cpu().numpy().astype(np.int64) for x in (batch.tok_seq, batch.tok_pos))
        table = self.cache.page_table.cpu().numpy()
        assert np.array_equal(table, self.cache.book.table)
        sc = types.SimpleNamespace(dtype=self.dtype, d=self.d, kv=self.kv, hq=self.hq, table=table, n_ids=n_ids)
        for layer in range(self.layers):
            q, k, v = self.rand(T, self.hq, self.d), self.rand(T, self.kv, self.d), self.rand(T, self.kv, self.d)
            out, lse = self.pipe.step(layer, batch, q, k, v, prefixes=px, weights=self.weights[layer])
            torch.cuda.synchronize()
            pages = np.concatenate((self.cache.pool.pages[layer].cpu().numpy(), self.cache.pool.cold[layer].numpy()))
            kp, vp = U.page_values(pages, self.d)
            lists = None
            if self.routed:
                n_list = self.hga.hga_token_list_size(self.plan)
                lists = self.pipe._buffer("lists", (T, self.kv, n_list), torch.int32).cpu().numpy()
            ref, rlse, mag, reach, count = U.attend(f64(q), kp, vp, table, seq, pos, self.kv, lists, n_ids)
            if px is None:
                tol, ltol = U.attend_tolerance(self.dtype, self.d, ref, mag, reach, count)
            else:
                tol, ltol = P.attend_tolerance(sc, ref, mag, reach, count, vp, seq, pos)
            assert (np.abs(f64(out) - ref) <= tol).all() and (np.abs(f64(lse) - rlse) <= ltol).all()
            # what each step adds, on what the steps before left
            self.want[layer], tol = P.weigh(f64(q), f64(lse), kp, table, seq, pos, self.kv, lists, n_ids, self.want[layer])
            self.tol[layer] += tol
            assert (np.abs(f64(self.weights[layer]) - self.want[layer]) <= self.tol[layer]).all()
        return px

    def evict(self, budget):
        total = self.weights.sum(0)
        book = self.cache.book
        n = len(book.length)
        want = np.broadcast_to(np.asarray(budget, np.int64), (n,))
        ref = P.choose(book.table, book.n_pages + book.n_cold, book.length, total.cpu().numpy(), want, 24, 1, 2)
        got = self.cache.evict(total, budget)
        assert got == [[c for c in row if c >= 0] for row in ref.tolist()]
        assert np.array_equal(self.cache.page_table.cpu().numpy(), book.table)
        return got


@pytest.mark.parametrize("dtype,d,kv,ratio,routed", [("bf16", 128, 2, 4, False), ("f32", 64, 2, 3, False),
                                                     ("bf16", 64, 1, 8, False), ("bf16", 64, 2, 2, True),
                                                     ("f32", 128, 1, 4, True)])
def test_samples_served_weighed_and_evicted(hga, dtype, d, kv, ratio, routed):
    t = _Served(hga, dtype, d, kv, ratio, routed)
    cache = t.cache
    assert t.serve([0, 4], [64 * 12 + 20, 100]) is None
    for s in (1, 2, 3):
        cache.fork(0, s)
    px = t.serve([3, 0, 4, 1, 2], [1, 2, 1, 1, 40])
    if not routed:
        assert px.n_groups == 1 and px.group_pages.tolist() == [12] and px.group_begin.tolist() == [0, 44]
        assert px.order.tolist() == [0, 1, 2, *range(4, 45), 3] and px.shared_hint == 12
    # each sequence of the prompt down to nine pages: their weights differ, so the prompts' pages do too
    gone = t.evict([9, 9, 9, 9, 9, 9])
    assert [len(x) for x in gone] == [4, 4, 4, 4, 0, 0] and cache.evict(t.weights[0], 20) == [[] for _ in range(6)]
    t.serve([0, 1, 2, 3], [1, 1, 1, 1])
    cache.fork(2, 5)
    cache.to_cold(2, 0, 1)
    px = t.serve([5, 2, 1], [3, 1, 1])
    if not routed:
        assert px.n_groups >= 1
    assert t.evict(0)[5]
    cache.compact()
    t.serve([0, 1, 2, 3, 4, 5], [1, 70, 1, 1, 1, 1])
    t.serve([0], [1], share=False)
    if routed:
        with pytest.raises(hga.HgaError):
            batch = cache.append([1], [1])
            one = P.i32([0])
            t.pipe.step(0, batch, t.rand(1, t.hq, d), t.rand(1, kv, d), t.rand(1, kv, d),
                        prefixes=hga.Prefixes(one, P.i32([0, 1]), one))
    for bad in (lambda: cache.prefixes(hga.TokenBatch(P.i32([0]), P.i32([0]), cache.page_table), [0], [2]),
                lambda: cache.book.evict(0, [23])):
        with pytest.raises(ValueError):
            bad()


def test_a_captured_step_over_shared_pages(hga):
    """A decode step with prefixes and weights captured, replayed for the next
    tokens, against a pipeline that runs each."""
    from paper_2606_30709_amd.pages import PagedCache
    from paper_2606_30709_amd.pipeline import TokenPipeline
    plan = hga.Plan(batch=1, n_q_heads=8, n_kv_heads=2, head_dim=128, keep_first=1, keep_last=1, topk_chunks=3,
                    topk_groups=4)
    cache = PagedCache(plan, 260, 24, 160, n_layers=1)
    pipe, other = TokenPipeline(cache, False), TokenPipeline(cache, False)
    g = torch.Generator().manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731
    pipe.step(0, cache.append([0], [64 * 145 + 5]), rand(9285, 8, 128), rand(9285, 2, 128), rand(9285, 2, 128))
    for s in range(1, 24):   # (so many that sharing pays)
        cache.fork(0, s)
    seqs, ones = list(range(24)), [1] * 24
    batch = cache.append(seqs, ones)
    px = cache.prefixes(batch, seqs, ones)
    q, k, v = rand(24, 8, 128), rand(24, 2, 128), rand(24, 2, 128)
    w, w2 = (torch.zeros(24, 2, 160, device="cuda") for _ in range(2))
    pipe.step(0, batch, q, k, v, px, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = pipe.step(0, batch, q, k, v, px, w)
    w.zero_()
    for _ in range(70):
        b = cache.append(seqs, ones)
        batch.tok_seq.copy_(b.tok_seq)
        batch.tok_pos.copy_(b.tok_pos)
        for x in (q, k, v):
            x.copy_(rand(*x.shape))
        graph.replay()
        want = other.step(0, batch, q, k, v, px, w2)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(w, w2)
    with pytest.raises(hga.HgaError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            TokenPipeline(cache, False).step(0, batch, q, k, v, px, w)
