"""Shared prefixes, page weights and evictions in 64 bits, written from
include/hga.h, over the scenes of tokens_util."""

from __future__ import annotations

import numpy as np
import torch

import tokens_util as U
from tokens_util import PAGE, f64


def i32(x):
    return torch.tensor(np.asarray(x, np.int32)).cuda()


def share(sc, groups):
    """Makes the sequences of each group (first row, other rows, pages) share
    the first row's leading pages."""
    for first, others, pages in groups:
        sc.table[others, :pages] = sc.table[first, :pages]


def prefixes(hga, seq, group_of_seq, pages, rng, shared_hint=None, own_hint=0):
    """Slots by group, in a random order inside each; sequences that are in none
    at either end."""
    seq = np.asarray(seq)
    of = np.array([group_of_seq.get(int(s), -1) for s in seq])
    G = len(pages)
    members = [rng.permutation(np.nonzero(of == g)[0]) for g in range(G)]
    rest = rng.permutation(np.nonzero(of < 0)[0])
    front = rest[:len(rest) // 3]
    order = np.concatenate([front, *members, rest[len(rest) // 3:]])
    begin = len(front) + np.concatenate([[0], np.cumsum([len(m) for m in members])])
    hint = max(list(pages) + [0]) if shared_hint is None else shared_hint
    return hga.Prefixes(i32(order), i32(begin), i32(pages), hint, own_hint)


def sharing(sc, batch, px, few=False):
    """The batch and prefixes with which the call shares whatever there is to
    share: through a table so wide, its hints unknown, that it looks worth it --
    and, where groups have more than 64 columns, worth the form for many of them
    (few: the one for few)."""
    columns = batch.n_tokens * (sc.hq // sc.kv)
    width = 600 if batch.n_tokens * sc.kv >= 90 else 4096
    if columns > 64 * px.n_groups > 0 and not few:
        width = max(batch.max_pages, -(-(3 << 15) // (columns // 16 * sc.kv)))
    wide = torch.full((batch.n_seqs, width), -1, dtype=torch.int32, device="cuda")
    wide[:, :batch.max_pages] = batch.page_table
    return (sc.hga.TokenBatch(batch.tok_seq, batch.tok_pos, wide),
            sc.hga.Prefixes(px.order, px.group_begin, px.group_pages, 0, px.own_hint))


def attend(sc, batch, px, q, workspace=True, stream=None, share=True):
    """The call, made to share (True; "few": in the form for few columns) or as
    it is.  workspace: True, or bytes, or a share of what it asks for."""
    hga = sc.hga
    if share:
        batch, px = sharing(sc, batch, px, share == "few")
    out = torch.full((batch.n_tokens, sc.hq, sc.d), float("nan"), dtype=U.DT[sc.dtype], device="cuda")
    lse = torch.full((batch.n_tokens, sc.hq), float("nan"), device="cuda")
    nb = hga.hga_attend_shared_workspace(sc.plan, batch, px)
    nb = nb if workspace is True else int(nb * workspace) // 16 * 16 if isinstance(workspace, float) else workspace
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
    hga.hga_attend_shared(sc.plan, sc.pool, sc.layer, batch, px, q, out, lse=lse, workspace=ws, stream=stream)
    return out, lse


def attend_tolerance(sc, ref, mag, reach, count, v, seq, pos):
    """Bounds as tokens_util.attend_tolerance's, but for bf16's weights, which
    enter as f16: 2^-11 of each for their rounding, and 2^-34 of the column's
    largest (two waves' share of 2^-35) where that is more -- of the sum of a
    token's |v| in all, for the weights come to at least the largest."""
    tol, ltol = U.attend_tolerance(sc.dtype, sc.d, ref, mag, reach, count)
    if sc.dtype == "bf16":
        exact = U.attend_tolerance("f32", sc.d, ref, mag, reach, count)[0]
        every = np.zeros_like(ref)
        for t, (s, p) in enumerate(zip(seq, pos)):
            if not count[t].any():
                continue
            ids = [i for i in sc.table[s, :p // PAGE + 1] if 0 <= i < sc.n_ids]
            every[t] = np.abs(np.nan_to_num(v[ids])).sum((0, 2)).repeat(sc.hq // sc.kv, 0)
        tol = exact + 2.0 ** -11 * mag + 2.0 ** -8 * np.abs(ref) + 2.0 ** -34 * every
    return tol, ltol


def check_attend(sc, q, got, tokens=slice(None)):
    """Against the definition of attention over each token's own row."""
    out, lse = got
    k, v = sc.k_v()
    seq, pos = sc.seq[tokens], sc.pos[tokens]
    ref, rlse, mag, reach, count = U.attend(f64(q)[tokens], k, v, sc.table, seq, pos, sc.kv, None, sc.n_ids)
    tol, ltol = attend_tolerance(sc, ref, mag, reach, count, v, seq, pos)
    o, l = f64(out)[tokens], f64(lse)[tokens]
    none = count == 0
    assert (o[none] == 0).all() and (l[none] == -np.inf).all()
    assert np.isfinite(o).all() and np.isfinite(l[~none]).all()
    err, lerr = np.abs(o - ref), np.abs(l[~none] - rlse[~none])
    assert (err <= tol).all(), float((err / tol).max())
    assert (lerr <= ltol[~none]).all(), float((lerr / ltol[~none]).max())


def weigh(q, lse, k, table, seq, pos, kv, lists, n_ids, prev):
    """weights and a bound on their error.  u = 2^-24.  A score is off by
    (d + 12) u reach, reach = sum |q||k| / sqrt(d) (see attend_tolerance); its
    exponent's argument log2(e) (s - lse) by 2 u (reach + |lse|) more, from its
    factors and lse's own: a weight p is off by p times the sum of both (and 4 u
    in exp2).  Each of a sum's terms is rounded into sums of at most all of them:
    rows, columns and tokens add (64 + tokens * heads + lists) u of the total."""
    T, hq, d = q.shape
    r, u = hq // kv, 2.0 ** -24
    out, tol = prev.astype(np.float64).copy(), np.zeros(prev.shape)
    terms = np.zeros(prev.shape)
    for t in range(T):
        if not (0 <= seq[t] < table.shape[0] and 0 <= pos[t] and pos[t] // PAGE < table.shape[1]):
            continue
        own, ids = pos[t] // PAGE, table[seq[t]]
        for h in range(kv):
            for c in (range(own + 1) if lists is None else lists[t, h]):
                if not (0 <= c <= own and 0 <= ids[c] < n_ids):
                    continue
                kk = k[ids[c], h, :pos[t] % PAGE + 1 if c == own else PAGE]
                for i in range(h * r, (h + 1) * r):
                    if not np.isinf(lse[t, i]):
                        s = kk @ q[t, i] / np.sqrt(d)
                        reach = np.abs(kk) @ np.abs(q[t, i]) / np.sqrt(d)
                        p = np.exp(s - lse[t, i])
                        out[seq[t], h, c] += p.sum()
                        tol[seq[t], h, c] += (p * ((d + 14) * u * reach + 2 * u * abs(lse[t, i]) + 8 * u)).sum()
                        terms[seq[t], h, c] += 1
    tol += (64 + 2 * terms + 4) * u * np.abs(out - prev) + (terms + 1) * u * np.abs(out)
    return out, tol + 1e-37


def run_weigh(sc, batch, q, lse, prev=None, lists=None, alias=False, workspace=True, stream=None):
    hga = sc.hga
    w = prev if alias else torch.full((batch.n_seqs, sc.kv, batch.max_pages), float("nan"), device="cuda")
    nb = hga.hga_weigh_pages_workspace(sc.plan, batch, lists) if workspace else 0
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
    hga.hga_weigh_pages(sc.plan, sc.pool, sc.layer, batch, q, lse, w, prev=prev, chunk_list=lists, workspace=ws,
                        stream=stream)
    return w


def check_weigh(sc, q, lse, got, prev=None, lists=None):
    p = np.zeros(tuple(got.shape)) if prev is None else f64(prev)
    ln = None if lists is None else lists.cpu().numpy()
    want, tol = weigh(f64(q), f64(lse), sc.k_v()[0], sc.table, sc.seq, sc.pos, sc.kv, ln, sc.n_ids, p)
    err = np.abs(f64(got) - want)
    assert (err <= tol).all(), float(np.nanmax(err / tol))


def choose(table, n_ids, seq_len, weights, budget, n_evict, first, window):
    out = np.full((table.shape[0], n_evict), -1, np.int32)
    for s in range(table.shape[0]):
        if not 0 < seq_len[s] <= table.shape[1] * PAGE:
            continue
        last = (seq_len[s] - 1) // PAGE
        here = [c for c in range(last + 1) if 0 <= table[s, c] < n_ids]
        may = np.array([c for c in here if first <= c < last - window], int)
        n = min(max(len(here) - int(budget[s]), 0), len(may), n_evict)
        with np.errstate(invalid="ignore"):
            total = sum((weights[s, h, may].astype(np.float64) for h in range(1, weights.shape[1])),
                        weights[s, 0, may].astype(np.float64))
        total = np.where(np.isnan(total), -np.inf, total)
        number = ~np.isnan(weights[s][:, may].astype(np.float64).sum(0))
        pick = may[np.lexsort((may, total, number))[:n]]
        out[s, :n] = np.sort(pick)
    return out


def run_choose(hga, plan, table, n_ids, seq_len, weights, budget, n_evict, stream=None):
    t, w = i32(table), torch.as_tensor(weights, device="cuda")
    out = torch.full((len(table), n_evict), -7, dtype=torch.int32, device="cuda")
    nb = hga.hga_choose_evictions_workspace(plan, t)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
    hga.hga_choose_evictions(plan, t, n_ids, i32(seq_len), w, i32(budget), out, workspace=ws, stream=stream)
    return out.cpu().numpy()
