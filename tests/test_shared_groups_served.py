"""Two groups of samples served through PagedCache and TokenPipeline in steps that
share their pages, one of the prompts evicted from and one partly in the cold
tier, against 64-bit definitions over what the pages hold."""

from __future__ import annotations

import types

import numpy as np
import pytest
import torch

import prefix_util as P
import tokens_util as U
from tokens_util import PAGE, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


@pytest.mark.parametrize("dtype,d,kv,ratio", [("bf16", 64, 2, 2), ("f32", 64, 2, 1), ("bf16", 128, 2, 4)])
def test_steps_that_share(hga, dtype, d, kv, ratio):
    from paper_2606_30709_amd.pages import PagedCache
    from paper_2606_30709_amd.pipeline import TokenPipeline
    hq, n = kv * ratio, 12
    plan = hga.Plan(batch=1, n_q_heads=hq, n_kv_heads=kv, head_dim=d, keep_first=1, keep_last=2, topk_chunks=3,
                    topk_groups=4, dtype=hga.F32 if dtype == "f32" else hga.BF16)
    cache = PagedCache(plan, 260, 2 * n + 1, 80, n_cold=12)
    pipe = TokenPipeline(cache, False)
    weights = torch.zeros(2 * n + 1, kv, 80, device="cuda")
    rng = np.random.default_rng(d + kv + ratio)
    rand = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(U.DT[dtype]).cuda()  # noqa: E731

    def serve(seqs, counts, check=True):
        batch = cache.append(seqs, counts)
        px = cache.prefixes(batch, seqs, counts)
        q, k, v = (rand(batch.n_tokens, h, d) for h in (hq, kv, kv))
        before = f64(weights)
        out, lse = pipe.step(0, batch, q, k, v, prefixes=px, weights=weights)
        if not check:
            return px
        # below its border the call would ask for the workspace of the tokens' own
        assert hga.hga_attend_shared_workspace(plan, batch, px) != hga.hga_attend_tokens_workspace(plan, batch)
        torch.cuda.synchronize()
        pages = np.concatenate((cache.pool.pages[0].cpu().numpy(), cache.pool.cold[0].numpy()))
        kp, vp = U.page_values(pages, d)
        table, n_ids = cache.book.table, cache.book.n_pages + cache.book.n_cold
        assert np.array_equal(cache.page_table.cpu().numpy(), table)
        seq, pos = (x.cpu().numpy().astype(np.int64) for x in (batch.tok_seq, batch.tok_pos))
        ref, rlse, mag, reach, count = U.attend(f64(q), kp, vp, table, seq, pos, kv, None, n_ids)
        sc = types.SimpleNamespace(dtype=dtype, d=d, kv=kv, hq=hq, table=table, n_ids=n_ids)
        tol, ltol = P.attend_tolerance(sc, ref, mag, reach, count, vp, seq, pos)
        assert (np.abs(f64(out) - ref) <= tol).all() and (np.abs(f64(lse) - rlse) <= ltol).all()
        want, tol = P.weigh(f64(q), f64(lse), kp, table, seq, pos, kv, None, n_ids, before)
        assert (np.abs(f64(weights) - want) <= tol).all()
        return px

    serve([0, n], [PAGE * 62 + 9, PAGE * 54 + 40], check=False)
    for s in range(1, n):
        cache.fork(0, s)
        cache.fork(n, n + s)
        for a in (0, n):
            weights[a + s] = weights[a]
    seqs = rng.permutation(2 * n).tolist()
    px = serve(seqs, [1] * 2 * n)
    assert sorted(px.group_pages.tolist()) == [54, 62] and px.shared_hint == 62
    # all samples of the first prompt give up the same pages, which are free then and absent of all
    free = cache.book.n_free()
    row = weights[:n].sum(0, keepdim=True)
    weights[:n] = row
    gone = cache.evict(weights, [50] * n + [80] * (n + 1))
    assert len(gone[0]) == 13 and all(g == gone[0] for g in gone[:n]) and not any(gone[n:])
    assert cache.book.n_free() == free + 13
    assert cache.to_cold(n + 3, 7, 19) == 12
    cache.append([2 * n], [70])     # one that shares nothing
    cache.release(2 * n)
    px = serve([2 * n, *seqs], [1] * (2 * n + 1))
    assert sorted(px.group_pages.tolist()) == [54, 62] and px.group_begin.tolist()[-1] == 2 * n
    cache.compact()
    serve(seqs, [1] * 2 * n)
