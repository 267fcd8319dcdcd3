"""hga_attend_shared where scores are so large that a reference's rounding shows
in the weights."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import prefix_util as P
import tokens_util as U
from tokens_util import PAGE, Scene, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


def _large(hga, dtype, d, kv, ratio, n, power, seed):
    """n sequences after one prompt of 21 pages; the largest |score| of a history
    is about 2^power in log2 units, and most histories have one key far ahead of
    all others.  The prompt's first pages hold smaller keys than its later ones."""
    lens = [PAGE * 21 + 1 + i * 69 // max(n - 1, 1) for i in range(n)]
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=seed)
    P.share(sc, [(0, list(range(1, n)), 21)])
    _, ks, _, _ = U.addresses(d)
    low = 127 + power // 2
    for c, page in enumerate(sc.table[0, :21]):
        e = sc.bytes[page][:, ks]
        sc.bytes[page][:, ks] = np.where(e == 255, 255, low - 40 + min(2 * c, 40))
    for s in range(n):
        page = sc.table[s, 21]
        e = sc.bytes[page][:, ks]
        sc.bytes[page][:, ks] = np.where(e == 255, 255, low)
    sc.pool.pages[0].copy_(torch.from_numpy(sc.bytes))
    q = sc.random(n, sc.hq, d, scale=2.0 ** (power - power // 2 - 4))
    return sc, q


@pytest.mark.parametrize("power", [20, 24, 25, 26, 27, 28, 29])
@pytest.mark.parametrize("dtype,d,kv,ratio,n,few", [
    ("bf16", 128, 2, 8, 30, False), ("bf16", 128, 2, 8, 30, "few"), ("bf16", 64, 1, 3, 60, False),
    ("bf16", 64, 2, 2, 5, "few"), ("f32", 64, 1, 16, 12, False), ("f32", 128, 2, 4, 6, "few")])
def test_scores_of_any_size(hga, dtype, d, kv, ratio, n, few, power):
    """A score s is off by (d + 12) 2^-24 reach (prefix_util), reach = the largest
    sum |q||k| / sqrt(d) of the row's: where the largest score is ahead of the
    next by 60 more than two of those, every other weight is below e^-60 of its
    own, all of them (1,400 at most, |v| <= 2^10) below 2^-60 in a result: the
    result is the key's value -- rounded once in bf16 (2^-8), off by 2^-22 in
    fp32 (three terms of a weight, the quotient) -- and lse lies between the
    score and that plus the log of the number of keys, off by the score's error
    and 4 2^-24 of itself (the factor to natural units, its product, the sum)."""
    sc, q = _large(hga, dtype, d, kv, ratio, n, power, seed=power + n)
    seq = np.arange(n)
    pos = np.array([sc.lens[s] - 1 for s in seq])
    batch = sc.batch(seq, pos)
    px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [21], sc.rng, own_hint=2)
    out, lse = (f64(x) for x in P.attend(sc, batch, px, q, share=few or True))
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    k, v = sc.k_v()
    u, ahead = 2.0 ** -24, 0
    largest = 0.0
    for t in range(n):
        ids = sc.table[seq[t], :pos[t] // PAGE + 1]
        for i in range(sc.hq):
            kk, vv = (x[ids, i // ratio].reshape(-1, d)[:pos[t] + 1] for x in (k, v))
            qi = f64(q[t, i])
            s = kk @ qi / np.sqrt(d)
            reach = (np.abs(kk) @ np.abs(qi)).max() / np.sqrt(d)
            off = (d + 12) * u * reach
            first, second = np.sort(s)[::-1][:2]
            largest = max(largest, abs(first) * np.log2(np.e))
            assert abs(lse[t, i] - first) <= off + 4 * u * abs(first) + np.log(len(s)) + 1e-5
            if first - second > 2 * off + 60:
                ahead += 1
                want = vv[s.argmax()]
                rel = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
                assert (np.abs(out[t, i] - want) <= rel * np.abs(want) + 2.0 ** -60).all()
    assert ahead >= n * sc.hq // 2 and 2.0 ** (power - 2) < largest < 2.0 ** 30.5


@pytest.mark.parametrize("dtype,d,kv,ratio,n", [("bf16", 128, 2, 8, 30), ("bf16", 64, 1, 3, 60), ("bf16", 128, 1, 4, 3), ("f32", 64, 1, 1, 90)])
@pytest.mark.parametrize("few", [False, "few"])
def test_queries_of_idle_tokens_change_no_bit_of_the_others(hga, dtype, d, kv, ratio, n, few):
    """Padding slots among a group's, whose queries are zeros, the largest numbers,
    infinities or NaN."""
    lens = [PAGE * 17 + 1 + i for i in range(n)]
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=n)
    P.share(sc, [(0, list(range(1, n)), 17)])
    seq = np.array([0, 1, -1, n, *range(n)])
    pos = np.array([-1, 10 ** 7, 5, 5] + [x - 1 for x in lens])
    batch = sc.batch(seq, pos)
    order = sc.rng.permutation(n + 4)
    px = hga.Prefixes(P.i32(order), P.i32([0, n + 4]), P.i32([17]), 17, 2)
    q = sc.random(n + 4, sc.hq, d)
    got = []
    for x in (0.0, torch.finfo(q.dtype).max, -torch.finfo(q.dtype).max, float("inf"), float("nan")):
        q[:4] = x
        got.append(P.attend(sc, batch, px, q, share=few or True))
        assert all(torch.equal(a, b) for a, b in zip(got[0], got[-1])), x
    assert (got[0][0][:4] == 0).all() and (got[0][1][:4] == -float("inf")).all()
    P.check_attend(sc, q, got[0], tokens=np.arange(4, n + 4, 4))
