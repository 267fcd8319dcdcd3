"""Shared prefixes, page weights and evictions where they can go wrong: values
that are no numbers or too large for a product's type, absent stretches, idle
tokens, streams, captured calls, refusals."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import prefix_util as P
import tokens_util as U
from tokens_util import PAGE, Scene, f64

pytestmark = pytest.mark.gpu

# columns of a group: few, some and many of them
SHAPES = [("bf16", 128, 2, 8, 3), ("bf16", 128, 1, 8, 7), ("bf16", 128, 2, 8, 30), ("bf16", 64, 2, 2, 5),
          ("bf16", 64, 1, 3, 60), ("f32", 128, 2, 4, 20), ("f32", 64, 1, 1, 90), ("f32", 64, 2, 5, 4)]


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def _same(a, b):
    return all(torch.equal(_bits(x), _bits(y)) for x, y in zip(a, b))


def _group(hga, dtype, d, kv, ratio, n, pages, seed=0, extra=1, tail=70):
    """n sequences after one prompt of `pages` pages, `extra` that share nothing."""
    lens = [PAGE * pages + 1 + i * (tail - 1) // max(n - 1, 1) for i in range(n)] + [100] * extra
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=seed)
    P.share(sc, [(0, list(range(1, n)), pages)])
    return sc


def _upload(sc):
    sc.pool.pages[0].copy_(torch.from_numpy(sc.bytes[:sc.pool.pages.shape[1]]))


@pytest.mark.parametrize("dtype,d,kv,ratio,n", SHAPES)
def test_values_that_are_no_numbers(hga, dtype, d, kv, ratio, n):
    """Value blocks that stand for NaN in a shared page, in a token's own and in
    one that some tokens of the group end inside of: the tokens that see the row
    are NaN in the block's dimensions, and nothing else is."""
    pages = 21
    sc = _group(hga, dtype, d, kv, ratio, n, pages, seed=n)
    _, _, _, vs = U.addresses(d)
    clean = sc.k_v()
    seq = np.array([*range(n + 1), 0, n - 1, 1])
    inside = np.array([5 * PAGE + 40, 5 * PAGE + 9, 17])     # three more tokens inside the prefix
    for late in (False, True):
        pos = np.array([sc.lens[s] - 1 for s in range(n + 1)] + (list(inside) if not late else [PAGE * pages] * 3))
        batch = sc.batch(seq, pos)
        q = sc.random(len(seq), sc.hq, d)
        bad = [(0, 5 * PAGE + 20, 0, 0), (n - 1, PAGE * pages, kv - 1, d // 32 - 1), (0, 3 * PAGE, kv - 1, 1)]
        want = np.zeros((len(seq), sc.hq, d), bool)
        before = sc.bytes.copy()
        for s, p, h, b in bad:
            page = sc.table[s, p // PAGE]
            sc.bytes[page, h, int(vs[p % PAGE, 32 * b])] = 255
            for t in range(len(seq)):
                if sc.table[seq[t], p // PAGE] == page and pos[t] >= p:
                    want[t, h * ratio:(h + 1) * ratio, 32 * b:32 * b + 32] = True
        _upload(sc)
        px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], sc.rng)
        ref, rlse, mag, reach, count = U.attend(f64(q), *clean, sc.table, seq, pos, kv, None, sc.n_ids)
        tol, ltol = P.attend_tolerance(sc, ref, mag, reach, count, clean[1], seq, pos)
        for share in (True, "few", False):
            out, lse = P.attend(sc, batch, px, q, share=share)
            o = f64(out)
            assert np.array_equal(np.isnan(o), want)
            err, lerr = (np.abs(o - ref) / tol)[~want].max(), (np.abs(f64(lse) - rlse) / ltol).max()
            assert err <= 1 and lerr <= 1
        sc.bytes[:] = before
        _upload(sc)


@pytest.mark.parametrize("dtype,d,kv,ratio,n", SHAPES)
@pytest.mark.parametrize("low,high", [(60, 66), (150, 180), (108, 141)])
def test_values_beyond_sixteen_bits(hga, dtype, d, kv, ratio, n, low, high):
    """Scales that f16 has no bits for, in one row of a shared page, in a whole
    one, and in a token's own."""
    pages = 19
    sc = _group(hga, dtype, d, kv, ratio, n, pages, seed=n + low)
    rng, first = sc.rng, PAGE * (d + d // 32)
    _, _, _, vs = U.addresses(d)
    sc.bytes[sc.table[0, 4]][:, vs[33]] = high
    sc.bytes[sc.table[0, 9]][:, first:] = rng.integers(low, high, sc.bytes[sc.table[0, 9]][:, first:].shape)
    sc.bytes[sc.table[n, 0]][:, vs[3]] = low
    _upload(sc)
    seq = np.arange(n + 1)
    batch = sc.batch(seq, [sc.lens[s] - 1 for s in seq])
    q = sc.random(n + 1, sc.hq, d)
    px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], rng)
    P.check_attend(sc, q, P.attend(sc, batch, px, q))


@pytest.mark.parametrize("dtype,d,kv,ratio,n", SHAPES)
@pytest.mark.parametrize("low,high", [(109, 112), (109, 141), (137, 141), (108, 110)])
def test_values_at_the_ends_of_sixteen_bits(hga, dtype, d, kv, ratio, n, low, high):
    """All values as small, or as large, as f16 holds them (its subnormals among
    them): a value that is lost there would be all of a result."""
    pages = 11
    sc = _group(hga, dtype, d, kv, ratio, n, pages, seed=n + low)
    first = PAGE * (d + d // 32)
    sc.bytes[..., first:] = sc.rng.integers(low, high, sc.bytes[..., first:].shape)
    _upload(sc)
    seq = np.arange(n + 1)
    batch = sc.batch(seq, [sc.lens[s] - 1 for s in seq])
    q = sc.random(n + 1, sc.hq, d)
    px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], sc.rng)
    P.check_attend(sc, q, P.attend(sc, batch, px, q))


@pytest.mark.parametrize("dtype,d,kv,ratio", [("bf16", 128, 2, 8), ("f32", 64, 1, 2), ("bf16", 64, 3, 1)])
def test_groups_of_very_different_sizes(hga, dtype, d, kv, ratio):
    """One large group among small ones and the other way round; prefixes of one
    page and of many."""
    for sizes, pages in (((70, 1, 2, 1, 3, 2, 2, 1), (9, 1, 40, 2, 3, 66, 5, 1)), ((1, 90, 1), (70, 20, 1)), ((2,) * 70, (3,) * 70)):
        lens, groups, at = [], [], 0
        for m, p in zip(sizes, pages):
            lens += [PAGE * p + 1 + 13 * i % 200 for i in range(m)]
            groups.append((at, list(range(at + 1, at + m)), p))
            at += m
        sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=len(sizes))
        P.share(sc, groups)
        seq = sc.rng.permutation(at)
        batch = sc.batch(seq, [lens[s] - 1 for s in seq])
        q = sc.random(at, sc.hq, d)
        of = {s: g for g, (a, more, _) in enumerate(groups) for s in [a, *more]}
        P.check_attend(sc, q, P.attend(sc, batch, P.prefixes(hga, seq, of, list(pages), sc.rng), q))


@pytest.mark.parametrize("dtype,d,kv,ratio,n", SHAPES)
def test_long_prefixes_with_absent_stretches(hga, dtype, d, kv, ratio, n):
    """Prefixes of a page more than 64, 128; more than 64 absent pages in a row;
    single pages between absent ones; any number of runs."""
    n = min(n, 20)
    for pages, gone in ((65, []), (129, [*range(5, 75), 80, 82, 84, 126, 127]), (70, [*range(1, 69)]), (66, [65]), (1, [])):
        sc = _group(hga, dtype, d, kv, ratio, n, pages, seed=pages)
        sc.table[:n, gone] = -1
        seq = np.arange(n + 1)
        batch = sc.batch(seq, [sc.lens[s] - 1 for s in seq])
        q = sc.random(n + 1, sc.hq, d)
        for hint in (None, 1, 9, 2 ** 31 - 1):
            px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], sc.rng, hint)
            P.check_attend(sc, q, P.attend(sc, batch, px, q, share=hint != 9))


@pytest.mark.parametrize("dtype,d,kv,ratio,n", SHAPES)
def test_idle_tokens_in_groups(hga, dtype, d, kv, ratio, n):
    """Idle tokens among a group's, beside a sequence's others, and whole units of
    them; queries of idle tokens may be anything."""
    pages = 13
    sc = _group(hga, dtype, d, kv, ratio, n, pages, seed=n + 5)
    seq = np.array([*range(n + 1)] + [0, 0, -1, n + 7] + [1, -3] * 70)
    pos = np.array([sc.lens[s] - 1 for s in range(n + 1)] + [-1, 10 ** 7, 5, 5] + [2 ** 31 - 1, 3] * 70)
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, d)
    q[n + 1:] = float("nan")
    T = len(seq)
    real = [*range(n + 1)]
    for order in (np.arange(T), sc.rng.permutation(T), np.arange(T)[::-1].copy()):
        # all but the sequence that shares nothing are in the group
        order = np.concatenate([order[order != n], [n]])
        px = hga.Prefixes(P.i32(order), P.i32([0, T - 1]), P.i32([pages]), pages, 2)
        out, lse = P.attend(sc, batch, px, q)
        assert (f64(out)[n + 1:] == 0).all() and (f64(lse)[n + 1:] == -np.inf).all()
        P.check_attend(sc, q, (out, lse), tokens=real)
        out, lse = P.attend(sc, batch, px, q, share="few")
        assert (f64(out)[n + 1:] == 0).all() and (f64(lse)[n + 1:] == -np.inf).all()
        P.check_attend(sc, q, (out, lse), tokens=real)
    # nothing but idle ones; no sequences, no pages in the table
    for shape in ((len(sc.lens), sc.max_pages), (0, 30), (3, 0), (0, 0)):
        b = hga.TokenBatch(torch.full_like(batch.tok_seq, -1), batch.tok_pos,
                           torch.zeros(shape, dtype=torch.int32, device="cuda"))
        sc.pool.pages[0, 0].fill_(255)
        out, lse = P.attend(sc, b, px, q)
        assert (f64(out) == 0).all() and (f64(lse) == -np.inf).all()
        w = P.run_weigh(sc, b, q, lse)
        assert (f64(w) == 0).all()
    empty = hga.TokenBatch(batch.tok_seq[:0], batch.tok_pos[:0], batch.page_table)
    px = hga.Prefixes(P.i32([]), P.i32([0, 0]), P.i32([5]))
    P.attend(sc, empty, px, q[:0])
    prev = torch.rand(len(sc.lens), kv, sc.max_pages, device="cuda")
    assert torch.equal(P.run_weigh(sc, empty, q[:0], lse[:0], prev), prev)


def test_groups_that_are_none(hga):
    """Words that the header does not allow: nothing outside the call is touched
    and the call comes back."""
    sc = _group(hga, "bf16", 64, 2, 4, 20, 6, seed=2)
    seq = np.arange(21)
    batch = sc.batch(seq, [sc.lens[s] - 1 for s in seq])
    q = sc.random(21, sc.hq, 64)
    big = 2 ** 31 - 1
    before = sc.stored()
    for order, begin, pages in (([0] * 21, [0, 21], [6]), ([-1, big, -big] * 7, [0, 21], [6]),
                                (np.arange(21), [30, -5, 7], [big, -big]), (np.arange(21), [5, 5, 5], [1, 2]),
                                (np.arange(21), [-big, big, 3, 12], [big, big, 6])):
        out = torch.full((23, sc.hq, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        b2, px = P.sharing(sc, batch, hga.Prefixes(P.i32(order), P.i32(begin), P.i32(pages)))
        nb = hga.hga_attend_shared_workspace(sc.plan, b2, px)
        ws = torch.full((nb + 64,), 7, dtype=torch.uint8, device="cuda")
        hga.hga_attend_shared(sc.plan, sc.pool, 0, b2, px, q, out[1:22], workspace=ws[:nb])
        torch.cuda.synchronize()
        assert (out[0] == 5).all() and (out[22] == 5).all() and (ws[nb:] == 7).all()
    assert np.array_equal(before, sc.stored())


@pytest.mark.parametrize("dtype,d,kv,ratio,n", [("bf16", 128, 2, 8, 20), ("f32", 64, 2, 2, 6)])
def test_streams_and_replayed_graphs(hga, dtype, d, kv, ratio, n):
    """A decode step over shared pages with its weights and evictions captured
    once: replayed with other queries, positions and groups, its workspaces filled
    with anything, beside the same calls on another stream with workspaces of
    their own."""
    pages = 40
    sc = _group(hga, dtype, d, kv, ratio, n, pages, seed=3)
    seq = np.arange(n + 1)
    batch = sc.batch(seq, [min(sc.lens[s] - 1, PAGE * pages) for s in seq])
    q = sc.random(n + 1, sc.hq, d)
    plain = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], sc.rng, own_hint=2)
    batch, px = P.sharing(sc, batch, plain)
    length, budget = batch.tok_pos + 1, torch.full((n + 1,), 30, dtype=torch.int32, device="cuda")

    def state():
        f = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        st = dict(out=torch.zeros_like(q), lse=f(n + 1, sc.hq), w=f(n + 1, kv, batch.max_pages),
                  ev=f(n + 1, 15, t=torch.int32))
        for name, nb in (("a", hga.hga_attend_shared_workspace(sc.plan, batch, px)),
                         ("b", hga.hga_weigh_pages_workspace(sc.plan, batch)),
                         ("c", hga.hga_choose_evictions_workspace(sc.plan, batch.page_table))):
            st["ws" + name] = f(max(nb, 16), t=torch.uint8)
        return st

    def calls(st):
        hga.hga_attend_shared(sc.plan, sc.pool, 0, batch, px, q, st["out"], lse=st["lse"], workspace=st["wsa"])
        hga.hga_weigh_pages(sc.plan, sc.pool, 0, batch, q, st["lse"], st["w"], prev=st["w"], workspace=st["wsb"])
        hga.hga_choose_evictions(sc.plan, batch.page_table, sc.n_ids, length, st["w"], budget, st["ev"],
                                 workspace=st["wsc"])

    names = ("out", "lse", "w", "ev")
    a, b, c = state(), state(), state()
    calls(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(a)
    side = torch.cuda.Stream()
    for i in range(5):
        q.copy_(sc.random(n + 1, sc.hq, d))
        batch.tok_pos.add_(-3 * i)
        length.copy_(batch.tok_pos + 1)
        if i == 3:   # other groups, a smaller prefix
            px.group_pages.fill_(17)
        for st in (a, b, c):
            st["w"].copy_(torch.arange(st["w"].numel(), device="cuda").view_as(st["w"]) % (7 + i))
            for w in "abc":
                st["ws" + w].fill_(255 - i)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):   # beside the replay
            calls(c)
        torch.cuda.synchronize()
        calls(b)
        for other in (b, c):
            assert _same([a[x] for x in names], [other[x] for x in names])
        sc.pos = batch.tok_pos.cpu().numpy().astype(np.int64)
        P.check_attend(sc, q, (a["out"], a["lse"]))


def test_refusals(hga):
    sc = _group(hga, "bf16", 64, 2, 2, 3, 4, seed=1)
    b = sc.batch([0, 1, 2], [260, 261, 262])
    q, lse = sc.random(3, 4, 64), torch.zeros(3, 4, device="cuda")
    out = torch.full_like(q, 3)
    w = torch.full((4, 2, sc.max_pages), 3.0, device="cuda")
    ev = torch.full((4, 2), 3, dtype=torch.int32, device="cuda")
    n4 = torch.full((4,), 100, dtype=torch.int32, device="cuda")
    px = P.prefixes(hga, [0, 1, 2], {0: 0, 1: 0, 2: 0}, [4], sc.rng)
    lists = torch.zeros(3, 2, 5, dtype=torch.int32, device="cuda")
    odd = torch.empty(3 * 4 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:769].view(3, 4, 64)
    att = lambda **x: hga.hga_attend_shared(sc.plan, sc.pool, x.get("layer", 0), b, x.get("px", px),  # noqa: E731
                                            x.get("q", q), x.get("out", out), lse=x.get("lse"), workspace=x.get("ws"))
    weigh = lambda **x: hga.hga_weigh_pages(sc.plan, sc.pool, x.get("layer", 0), b, x.get("q", q),  # noqa: E731
                                            x.get("lse", lse), x.get("w", w), prev=x.get("prev"),
                                            chunk_list=x.get("lists"), workspace=x.get("ws"))
    choose = lambda **x: hga.hga_choose_evictions(sc.plan, x.get("table", b.page_table), x.get("n_ids", 5),  # noqa: E731
                                                  x.get("len", n4), x.get("w", w), x.get("budget", n4),
                                                  x.get("ev", ev), workspace=x.get("ws"))
    few = hga.Prefixes(px.order[:2], px.group_begin, px.group_pages)
    bad = [(att, dict(layer=1)), (att, dict(layer=-1)), (att, dict(px=few)), (att, dict(q=odd)), (att, dict(out=odd)),
           (att, dict(out=out.float())), (att, dict(q=q[:2])), (att, dict(lse=lse[:, :3])), (att, dict(ws=odd.view(-1))),
           (weigh, dict(layer=1)), (weigh, dict(lse=lse[:2])), (weigh, dict(lse=lse.double())), (weigh, dict(w=w[:3])),
           (weigh, dict(w=w[..., :-1])), (weigh, dict(prev=w.half())), (weigh, dict(prev=w.cpu())),
           (weigh, dict(lists=lists[:2])), (weigh, dict(lists=lists.long())), (weigh, dict(lists=lists[..., :0])),
           (weigh, dict(q=odd)), (choose, dict(n_ids=-1)), (choose, dict(table=b.page_table.long())),
           (choose, dict(len=n4[:3])), (choose, dict(budget=n4.long())), (choose, dict(w=w[:, :1])),
           (choose, dict(w=w.transpose(1, 2))), (choose, dict(ev=ev[:3])), (choose, dict(ev=ev.t().contiguous().t()))]
    for f, kw in bad:
        with pytest.raises(hga.HgaError) as e:
            f(**kw)
        assert e.value.status in (-1, -2, -3), kw
    for make in (lambda: hga.Prefixes(px.order.long(), px.group_begin, px.group_pages),
                 lambda: hga.Prefixes(px.order, px.group_begin[:1], px.group_pages),
                 lambda: hga.Prefixes(px.order, px.group_begin, px.group_pages.cpu()),
                 lambda: hga.Prefixes(px.order.cpu(), px.group_begin.cpu(), px.group_pages.cpu()),
                 lambda: att(px=hga.Prefixes(px.order, px.group_begin, px.group_pages, -1)),
                 lambda: att(px=hga.Prefixes(px.order, px.group_begin, px.group_pages, 0, -1))):
        with pytest.raises(hga.HgaError):
            make()
    wide = torch.zeros(2, 17000, dtype=torch.int32, device="cuda")
    with pytest.raises(hga.HgaError):   # a workspace it cannot do without
        choose(table=wide, len=n4[:2], budget=n4[:2], ev=ev[:2], w=torch.zeros(2, 2, 17000, device="cuda"))
    torch.cuda.synchronize()
    assert (out == 3).all() and (w == 3).all() and (ev == 3).all()
    choose(ev=ev[:, :0])   # nothing to write
