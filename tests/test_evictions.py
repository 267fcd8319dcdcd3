"""Attention weights of pages and the choice of evictions against 64-bit
definitions (prefix_util)."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import prefix_util as P
from tokens_util import Scene, f64

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 128, 4, 8), ("f32", 128, 1, 16), ("bf16", 64, 3, 3), ("f32", 64, 2, 1), ("bf16", 64, 1, 16),
          ("bf16", 128, 5, 2), ("f32", 128, 2, 5), ("f32", 64, 3, 3)]


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


def _prev(sc):
    return torch.rand(len(sc.lens), sc.kv, sc.max_pages, device="cuda")


@pytest.mark.parametrize("dtype,d,kv,ratio", SHAPES)
def test_weights_of_whole_histories(hga, dtype, d, kv, ratio):
    lens = (1, 63, 64, 65, 130, 777, 2, 1600)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, layers=2, layer=1, seed=1, cold=9)
    sc.table[5, 2:6] = [-1, sc.n_ids, 2 ** 31 - 1, -2 ** 31]
    seq = [7, 1, 2, 3, 4, 5, 6, -1, 8, 5, 5, 7, 3]       # sequence 0 has no token here
    pos = [lens[s] - 1 for s in seq[:7]] + [3, 0, -1, 10 ** 7, 800, 64]
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, d, scale=1.5)
    lse = sc.attend(batch, q)[1]
    got = P.run_weigh(sc, batch, q, lse)
    P.check_weigh(sc, q, lse, got)
    # the tokens' heads' softmax weights come to one each
    total = f64(got).sum(-1)
    count = np.bincount([s for s, p in zip(seq, pos) if 0 <= s < 8 and 0 <= p < 64 * sc.max_pages], minlength=8)
    assert np.abs(total - ratio * count[:, None]).max() <= 1e-4 * ratio
    prev = _prev(sc)
    got = P.run_weigh(sc, batch, q, lse, prev)
    P.check_weigh(sc, q, lse, got, prev)
    assert torch.equal(got, P.run_weigh(sc, batch, q, lse, prev))
    assert torch.equal(got[0], prev[0]) and torch.equal(got, P.run_weigh(sc, batch, q, lse, prev.clone(), alias=True))
    wide = torch.zeros(len(seq), sc.hq + 3, d, dtype=q.dtype, device="cuda")
    wide[:, :sc.hq] = q
    assert torch.equal(got, P.run_weigh(sc, batch, wide[:, :sc.hq], lse, prev))
    P.check_weigh(sc, q, lse, P.run_weigh(sc, batch, q, lse, prev, workspace=False), prev)


@pytest.mark.parametrize("dtype,d,kv,ratio", SHAPES)
def test_weights_of_listed_pages(hga, dtype, d, kv, ratio):
    lens = (1, 64, 700, 1500, 129)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, cold=5, seed=2)
    sc.table[3, 4:9] = [-1, sc.n_ids, 2 ** 31 - 1, -2 ** 31, sc.table[3, 3]]
    seq = [0, 1, 2, 3, 4, 3, 3, 2, -1]
    pos = [0, 63, 699, 1499, 128, 700, 64, 640, 5]
    batch = sc.batch(seq, pos)
    lists = sc.rng.integers(-3, 26, (len(seq), kv, 9)).astype(np.int32)
    lists[6] = -1
    lists[3, 0] = [2 ** 31 - 1, -2 ** 31, 23, 23, 5, 8, 3, 0, 99]
    lt = torch.from_numpy(lists).cuda()
    q = sc.random(len(seq), sc.hq, d, scale=1.5)
    lse = sc.attend(batch, q, lt)[1]
    prev = _prev(sc)
    got = P.run_weigh(sc, batch, q, lse, prev, lt)
    P.check_weigh(sc, q, lse, got, prev, lt)
    assert torch.equal(got, P.run_weigh(sc, batch, q, lse, prev, lt))
    assert torch.equal(got, P.run_weigh(sc, batch, q, lse, prev.clone(), lt, alias=True))
    own = sc.route(batch, q)
    lse = sc.attend(batch, q, own)[1]
    P.check_weigh(sc, q, lse, P.run_weigh(sc, batch, q, lse, None, own), None, own)


@pytest.mark.parametrize("dtype,d,kv,ratio,new", [("bf16", 128, 1, 8, 40), ("f32", 64, 2, 1, 300), ("bf16", 64, 1, 3, 70)])
def test_weights_of_a_prompts_tokens(hga, dtype, d, kv, ratio, new):
    lens = (300, 64, 5, 900)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=4)
    runs = [(s, max(0, x - new), x) for s, x in enumerate(lens)]
    seq = np.concatenate([[s] * (b - a) for s, a, b in runs])
    pos = np.concatenate([np.arange(a, b) for _, a, b in runs])
    q = sc.random(len(seq), sc.hq, d)
    for o in (np.arange(len(seq)), sc.rng.permutation(len(seq))):
        batch = sc.batch(seq[o], pos[o])
        lse = sc.attend(batch, q)[1]
        prev = _prev(sc)
        P.check_weigh(sc, q, lse, P.run_weigh(sc, batch, q, lse, prev), prev)


def test_more_tokens_than_a_workgroup_looks_at_once(hga):
    """2,500 tokens of three sequences in turns, whole histories and lists."""
    lens = (200, 70, 130)
    sc = Scene(hga, "bf16", 64, 1, 2, lens=lens, seed=6)
    seq = np.arange(2500) % 3
    pos = sc.rng.integers(0, np.array(lens)[seq])
    batch = sc.batch(seq, pos)
    q = sc.random(2500, 2, 64)
    lse = sc.attend(batch, q)[1]
    prev = _prev(sc)
    P.check_weigh(sc, q, lse, P.run_weigh(sc, batch, q, lse, prev), prev)
    lists = torch.from_numpy(sc.rng.integers(0, 4, (2500, 1, 3)).astype(np.int32)).cuda()
    lse = sc.attend(batch, q, lists)[1]
    P.check_weigh(sc, q, lse, P.run_weigh(sc, batch, q, lse, prev, lists), prev, lists)


def test_a_head_without_a_finite_lse_adds_nothing(hga):
    sc = Scene(hga, "bf16", 128, 2, 4, lens=(500, 200), seed=7)
    batch = sc.batch([0, 1, 0], [499, 199, 70])
    q = sc.random(3, 8, 128)
    lse = sc.attend(batch, q)[1]
    lse[0, 1], lse[1, 5], lse[2] = -float("inf"), float("inf"), -float("inf")
    P.check_weigh(sc, q, lse, P.run_weigh(sc, batch, q, lse))


@pytest.mark.parametrize("kv,first,last", [(1, 1, 0), (4, 2, 8), (12, 0, 2)])
@pytest.mark.parametrize("n", [1, 7, 64, 200, 1500])
def test_chosen_pages(hga, kv, first, last, n):
    rng = np.random.default_rng(n + kv)
    S = 9
    plan = hga.Plan(batch=1, n_q_heads=kv, n_kv_heads=kv, head_dim=64, keep_first=first, keep_last=last, force_prev=1,
                    topk_chunks=4, topk_groups=4)
    table = rng.integers(-3, 5000, (S, n)).astype(np.int32)
    table[rng.random((S, n)) < 0.1] = 5000
    lens = rng.integers(1, 64 * n + 1, S)
    lens[:4] = [64 * n, 0, 64 * n + 1, -5]
    w = np.exp(4 * rng.standard_normal((S, kv, n))).astype(np.float32)
    w[:, :, rng.random(n) < 0.3] = 0            # ties
    w[3, :, ::2] = 1.5
    w[5] = 2.0
    w[6, 0, ::3] = np.nan
    w[7, 0, ::4], w[7, 0, 1::4] = np.inf, -np.inf
    w[8, 0, ::2] = -0.0
    for budget in (rng.integers(0, n + 2, S), np.zeros(S), np.full(S, 10 ** 9), np.full(S, -2 ** 31)):
        for most in (1, n, n + 3):
            got = P.run_choose(hga, plan, table, 5000, lens, w, budget, most)
            assert np.array_equal(got, P.choose(table, 5000, lens, w, budget, most, first, max(last, 1)))


@pytest.mark.parametrize("n", [1024, 1025, 4100, 16384, 16385, 40000])
def test_chosen_pages_of_long_tables(hga, n):
    """Keys in registers and in the workspace; equal ones in every place."""
    rng = np.random.default_rng(n)
    S, kv = 4, 2
    plan = hga.Plan(batch=1, n_q_heads=kv, n_kv_heads=kv, head_dim=64, keep_first=1, keep_last=3, force_prev=1,
                    topk_chunks=4, topk_groups=4)
    table = np.where(rng.random((S, n)) < 0.02, -1, rng.integers(0, 10 ** 6, (S, n))).astype(np.int32)
    lens = np.array([64 * n, 64 * n - 63, 64 * (n // 2) + 5, 64 * n - 7])
    w = np.exp(3 * rng.standard_normal((S, kv, n))).astype(np.float32)
    w[1] = rng.integers(0, 3, (kv, n))     # three values in all
    w[2] = 0.25                            # one
    w[3, 0], w[3, 1] = 1e30, rng.random(n)  # sums apart in their last bits, or not at all
    for budget in ([n // 4] * 4, [n - 20] * 4, [5] * 4, [n // 2, n // 3, 1, 0]):
        got = P.run_choose(hga, plan, table, 10 ** 6, lens, w, budget, n)
        assert np.array_equal(got, P.choose(table, 10 ** 6, lens, w, budget, n, 1, 3))


def test_weights_that_fp32_sums_cannot_tell_apart(hga):
    n = 400
    plan = hga.Plan(batch=1, n_q_heads=3, n_kv_heads=3, head_dim=64, keep_first=1, keep_last=0, force_prev=1,
                    topk_chunks=4, topk_groups=4)
    rng = np.random.default_rng(0)
    w = np.full((1, 3, n), 1000.0, np.float32)
    w[0, 2] = 1.0 + rng.permutation(n) * 2.0 ** -23
    args = (np.arange(n, dtype=np.int32)[None], n, [64 * n], w, [n // 3], n)
    assert np.array_equal(P.run_choose(hga, plan, *args), P.choose(*args, 1, 1))
