"""hga_attend_shared over runs of any length: more pages than a wavefront lists
at once, prefixes longer than the host said, fewer runs than the call asks for,
hundreds of groups.  Calls go with their hints as given."""

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


def _attend(q, k, v, table, seq, pos, kv, n_ids):
    """As tokens_util.attend over whole histories, a KV head's queries at a time."""
    T, hq, d = q.shape
    r = hq // kv
    out, mag = np.zeros((T, hq, d)), np.zeros((T, hq, d))
    lse, reach, count = np.full((T, hq), -np.inf), np.zeros((T, hq)), np.zeros((T, hq), int)
    for t in range(T):
        at = np.arange(pos[t] + 1)
        ids = table[seq[t], at // PAGE]
        here = (ids >= 0) & (ids < n_ids)
        for h in range(kv):
            kk, vv = (x[ids[here], h, at[here] % PAGE] for x in (k, v))
            heads = slice(h * r, (h + 1) * r)
            s = kk @ q[t, heads].T / np.sqrt(d)
            m = s.max(0)
            p = np.exp(s - m)
            l = p.sum(0)
            out[t, heads], mag[t, heads] = p.T @ vv / l[:, None], p.T @ np.abs(vv) / l[:, None]
            lse[t, heads] = m + np.log(l)
            reach[t, heads] = (np.abs(kk) @ np.abs(q[t, heads]).T).max(0) / np.sqrt(d)
            count[t, heads] = len(kk)
    return out, lse, mag, reach, count


class _Questions:
    """`seqs` sequences after one prompt of `pages` pages, `new` tokens of each:
    with 8,192 columns of two KV heads a hint of 96 pages is enough for the form
    for many columns."""

    def __init__(self, hga, dtype, d, ratio, pages, seed=0, gone=(), max_pages=None):
        self.hga, self.seqs, self.pages = hga, 4, pages
        self.new = 512 * 16 // ratio // 4
        lens = [PAGE * pages + self.new + 7 * i for i in range(4)]
        self.sc = sc = Scene(hga, dtype, d, 2, ratio, lens=lens, seed=seed, cold=5, max_pages=max_pages)
        P.share(sc, [(0, [1, 2, 3], pages)])
        sc.table[:, list(gone)] = -1
        self.seq = np.repeat(np.arange(4), self.new)
        self.pos = np.concatenate([np.arange(x - self.new, x) for x in lens])
        self.batch = sc.batch(self.seq, self.pos)
        self.q = sc.random(len(self.seq), sc.hq, d)

    def prefixes(self, hint, own):
        return P.prefixes(self.hga, self.seq, {s: 0 for s in range(4)}, [self.pages], self.sc.rng, hint, own)

    def least(self):
        """The workspace that holds one partial result of each kind."""
        T = len(self.seq)
        return -(-8 * T // 16) * 16 + 2 * T * self.sc.hq * (self.sc.d + 2) * 4

    def check(self, px, workspace):
        """Two tokens of each sequence against the definition."""
        sc = self.sc
        out, lse = P.attend(sc, self.batch, px, self.q, workspace=workspace, share=False)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        t = np.concatenate([[s * self.new + 5 * s, (s + 1) * self.new - 1] for s in range(4)])
        if not hasattr(self, "ref"):
            k, v = sc.k_v()
            ref, rlse, mag, reach, count = _attend(f64(self.q)[t], k, v, sc.table, self.seq[t], self.pos[t], sc.kv, sc.n_ids)
            tol, ltol = P.attend_tolerance(sc, ref, mag, reach, count, v, self.seq[t], self.pos[t])
            self.ref = ref, rlse, tol, ltol
        ref, rlse, tol, ltol = self.ref
        assert (np.abs(f64(out)[t] - ref) <= tol).all() and (np.abs(f64(lse)[t] - rlse) <= ltol).all()


FORMS = [("bf16", 128, 16), ("bf16", 64, 16), ("bf16", 128, 8), ("f32", 64, 16), ("f32", 128, 16)]


@pytest.mark.parametrize("dtype,d,ratio", FORMS)
@pytest.mark.parametrize("pages,gone", [(193, range(64, 128)), (130, [*range(3, 61), 63, 64, 129]), (257, [])])
def test_more_pages_in_a_run_than_are_listed_at_once(hga, dtype, d, ratio, pages, gone):
    t = _Questions(hga, dtype, d, ratio, pages, seed=pages, gone=gone)
    asked = t.least()
    for hint in (96, pages):
        px = t.prefixes(hint, 2)
        assert hga.hga_attend_shared_workspace(t.sc.plan, t.batch, px) >= asked
        t.check(px, asked)          # one run of each kind


@pytest.mark.parametrize("dtype,d,ratio", FORMS)
def test_prefixes_longer_than_the_host_said(hga, dtype, d, ratio):
    t = _Questions(hga, dtype, d, ratio, 203, seed=3, gone=[100, 101, 170])
    for hint, own, part in ((96, 1, True), (96, 4, 0.4), (150, 9, 0.7), (0, 0, True), (2 ** 31 - 1, 1, 0.5)):
        t.check(t.prefixes(hint, own), part)


@pytest.mark.parametrize("dtype,d,ratio", FORMS[:2])
@pytest.mark.parametrize("low,high", [(60, 66), (150, 180)])
def test_values_beyond_sixteen_bits_behind_the_first_pages_of_a_run(hga, dtype, d, ratio, low, high):
    t = _Questions(hga, dtype, d, ratio, 140, seed=low)
    _, _, _, vs = U.addresses(d)
    sc = t.sc
    sc.bytes[sc.table[0, 131]][:, vs[33]] = high
    sc.bytes[sc.table[0, 70]][:, vs[5]] = low
    sc.pool.pages[0].copy_(torch.from_numpy(sc.bytes[:sc.pool.pages.shape[1]]))
    sc.pool.cold[0].copy_(torch.from_numpy(sc.bytes[sc.pool.pages.shape[1]:]))
    t.check(t.prefixes(140, 3), t.least())
    t.check(t.prefixes(140, 3), True)


@pytest.mark.parametrize("dtype,d,kv,ratio,groups", [("bf16", 64, 2, 2, 500), ("f32", 64, 1, 1, 300), ("bf16", 128, 1, 8, 190)])
def test_hundreds_of_groups(hga, dtype, d, kv, ratio, groups):
    """Small groups among empty ones and ones that share nothing, in any number of
    64s; every token compared."""
    rng = np.random.default_rng(groups)
    sizes = rng.choice([0, 1, 2, 3, 3, 4], groups)
    pages = rng.integers(0, 4, groups)
    lens, rows, of = [], [], {}
    for g, (m, p) in enumerate(zip(sizes, pages)):
        at = len(lens)
        lens += [PAGE * int(p) + 1 + int(x) for x in rng.integers(0, 70, m)]
        rows.append((at, list(range(at + 1, at + m)), int(p)))
        of.update({s: g for s in range(at, at + m)})
    lens += [100, 1, 64]
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=groups)
    P.share(sc, [r for r, m in zip(rows, sizes) if m])
    seq = rng.permutation(len(lens))
    batch = sc.batch(seq, [lens[s] - 1 for s in seq])
    q = sc.random(len(seq), sc.hq, d)
    px = P.prefixes(hga, seq, of, pages.tolist(), rng, own_hint=2)
    wide = torch.full((max(len(lens), 2 * groups), 600), -1, dtype=torch.int32, device="cuda")
    wide[:len(lens), :batch.max_pages] = batch.page_table
    b = hga.TokenBatch(batch.tok_seq, batch.tok_pos, wide)
    px = hga.Prefixes(px.order, px.group_begin, px.group_pages, 600, 2)
    assert hga.hga_attend_shared_workspace(sc.plan, b, px) != hga.hga_attend_tokens_workspace(sc.plan, b)
    P.check_attend(sc, q, P.attend(sc, b, px, q, share=False))


def test_many_groups_of_many_columns(hga):
    """The form for many columns with more groups than a wavefront looks at once."""
    sizes = [1] * 60 + [300, 2, 1, 500] + [1] * 6
    pages = [2] * 60 + [9, 70, 1, 5] + [3] * 6
    new = [1] * 60 + [150, 1, 1, 250] + [1] * 6        # tokens of each of its (at most two) sequences
    lens, groups, runs, of = [], [], [], {}
    for g, (m, p, n) in enumerate(zip(sizes, pages, new)):
        at = len(lens)
        lens += [PAGE * p + n] * (m // n)
        groups.append((at, list(range(at + 1, len(lens))), p))
        for s in range(at, len(lens)):
            runs.append((s, n))
            of[s] = g
    sc = Scene(hga, "bf16", 64, 1, 8, lens=lens, seed=70)
    P.share(sc, groups)
    seq = np.concatenate([[s] * n for s, n in runs])
    pos = np.concatenate([np.arange(lens[s] - n, lens[s]) for s, n in runs])
    # rows that no token is of, so that there are two to a group
    more = np.full((150, sc.table.shape[1]), -1, np.int32)
    more[:len(lens)] = sc.table
    sc.table = more
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, 64)
    px = P.prefixes(hga, seq, of, pages, sc.rng)
    columns = len(seq) * 8
    assert columns > 64 * len(pages)
    P.check_attend(sc, q, P.attend(sc, batch, px, q), tokens=np.arange(0, len(seq), 5))
