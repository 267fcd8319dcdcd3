"""The paged 4-bit cache in 64 bits, written from include/hga.h: the stored
format, routing and attention of single tokens, and a scene of random pages."""

from __future__ import annotations

import numpy as np
import torch

PAGE = 64
MAG = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def quantise(x):
    """x [..., d] -> codes uint8 [..., d], scale bytes uint8 [..., d/32]."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    fin = np.isfinite(b).all(-1)
    amax = np.where(fin, np.abs(np.where(np.isfinite(b), b, 0)).max(-1), 0)
    s = np.full(amax.shape, -125)
    while (amax > 6 * 2.0 ** s).any():
        s += amax > 6 * 2.0 ** s
    s = np.minimum(s, 126)
    y = np.where(fin[..., None], np.abs(b), 0) / 2.0 ** s[..., None]
    dist = np.abs(y[..., None] - np.where(MAG > np.where(s == 126, 3, 6)[..., None, None], np.inf, MAG))
    best = dist.min(-1, keepdims=True)
    near = dist == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = np.where(fin[..., None], code + 8 * np.signbit(b), 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(fin, s + 127, 255).astype(np.uint8)


def values(codes, e):
    c = codes.reshape(*e.shape, 32).astype(int)
    sc = np.where(e == 255, np.nan, 2.0 ** (e.astype(float) - 127))
    return (np.where(c < 8, 1, -1) * MAG[c % 8] * sc[..., None]).reshape(codes.shape)


def head_bytes(d):
    return PAGE * d * 17 // 16


def addresses(d):
    """Byte of every element's code and of its scale, for keys and for values
    (the documented formulas), each [64, d]."""
    r, j = np.arange(PAGE)[:, None], np.arange(d)[None]
    half, dl, nb = 32 * d, d // 16, d // 32
    kc = r * (d // 2) + j // 2
    vc = half + (r // 4 * 16 + j // dl) * (4 * dl // 2) + r % 4 * (dl // 2) + j % dl // 2
    ks = 2 * half + (r % 16 * nb + j // 32) * 4 + r // 16
    vs = 2 * half + 64 * nb + ((r // 4 % 4 * nb + j // 32) * 4 + r // 16) * 4 + r % 4
    return kc, ks, vc, vs


def page_values(page, d):
    """Bytes [..., head_bytes] -> k, v [..., 64, d]."""
    kc, ks, vc, vs = addresses(d)
    hi = np.arange(d) % 2 * 4
    out = []
    for c, s in ((kc, ks), (vc, vs)):
        out.append(values(page[..., c] >> hi & 15, page[..., s][..., ::32]))
    return out


def write_row(page, d, row, k, v):
    """Row `row` of bytes [head_bytes] from k, v [d]."""
    kc, ks, vc, vs = addresses(d)
    for x, c, s in ((k, kc, ks), (v, vc, vs)):
        codes, e = quantise(x)
        page[c[row, ::2]] = codes[::2] | codes[1::2] << 4
        page[s[row, ::32]] = e


def summary(k, d, base, n_hf):
    """Mean of keys [..., 64, d] turned to the page's middle."""
    p = np.arange(d // 2)
    phi = np.where(p < n_hf, 0.0, ((PAGE - 1) / 2 - np.arange(PAGE))[:, None] * base ** (-2.0 * p / d))
    z = (k[..., :d // 2] + 1j * k[..., d // 2:]) * np.exp(1j * phi)
    z = z.mean(-2)
    return np.concatenate((z.real, z.imag), -1)


def f64(t):
    return t.detach().double().cpu().numpy()


def route(q, sums, table, seq, pos, kv, first, window, topk, n_list, n_ids):
    """Lists [T, kv, n_list] from q [T, Hq, d], sums [ids, kv, d]."""
    T, hq, d = q.shape
    qm = q.reshape(T, kv, hq // kv, d).sum(2)
    out = np.full((T, kv, n_list), -1, np.int32)
    for t in range(T):
        if not (0 <= seq[t] < table.shape[0] and 0 <= pos[t] and pos[t] // PAGE < table.shape[1]):
            continue
        own, ids = pos[t] // PAGE, table[seq[t]]
        has = [c for c in range(own + 1) if 0 <= ids[c] < n_ids]
        mid = np.array([c for c in has if first <= c < own - window], int)
        for h in range(kv):
            rest = [c for c in has if not first <= c < own - window]
            if len(mid):
                with np.errstate(invalid="ignore"):
                    s = (sums[ids[mid], h] * qm[t, h]).sum(-1)
                s = np.where(np.isnan(s), -np.inf, s)
                rest += list(mid[np.lexsort((mid, -s))[:topk]])
            out[t, h, :len(rest)] = sorted(rest)
    return out


def attend(q, k, v, table, seq, pos, kv, lists, n_ids):
    """out, lse and per-row error magnitudes: mag = sum p |v| / l and reach =
    the largest sum |q||k| / sqrt(d) of a row's scores.  k, v [ids, kv, 64, d]."""
    T, hq, d = q.shape
    r = hq // kv
    out, mag = np.zeros((T, hq, d)), np.zeros((T, hq, d))
    lse, reach, count = np.full((T, hq), -np.inf), np.zeros((T, hq)), np.zeros((T, hq), int)
    for t in range(T):
        if not (0 <= seq[t] < table.shape[0] and 0 <= pos[t] and pos[t] // PAGE < table.shape[1]):
            continue
        own, ids = pos[t] // PAGE, table[seq[t]]
        for h in range(kv):
            cs = range(own + 1) if lists is None else lists[t, h]
            cs = [c for c in cs if 0 <= c <= own and 0 <= ids[c] < n_ids]
            if not cs:
                continue
            kk, vv = (np.concatenate([x[ids[c], h, :pos[t] % PAGE + 1 if c == own else PAGE] for c in cs])
                      for x in (k, v))
            for i in range(h * r, (h + 1) * r):
                s = kk @ q[t, i] / np.sqrt(d)
                m = s.max()
                p = np.exp(s - m)
                l = p.sum()
                out[t, i], mag[t, i] = p @ vv / l, p @ np.abs(vv) / l
                lse[t, i] = m + np.log(l)
                reach[t, i] = (np.abs(kk) @ np.abs(q[t, i])).max() / np.sqrt(d)
                count[t, i] = len(kk)
    return out, lse, mag, reach, count


def attend_tolerance(dtype, d, out, mag, reach, count):
    """Bounds on |out error| and |lse error|.  u = 2^-24.  A score is a sum of d
    exact (bf16) or three-term products in fp32: off by (d + 8) u reach, and by
    4 u reach in its scaling and the exponent's argument; the maximum of a
    longer history is met by factors of as much.  With delta = twice that, a
    weight is off by delta (+ 4 u in exp2) relatively; the sums over the keys
    add count * u.  bf16 rounds each weight (half a step: 2^-8) and the result
    (2^-8 of it)."""
    u = 2.0 ** -24
    delta = 2 * (d + 12) * u * reach + 8 * u
    rel = 2 * delta + 2 * count * u + (2.0 ** -8 if dtype == "bf16" else 4 * u)
    tol = rel[..., None] * mag + (2.0 ** -8 if dtype == "bf16" else 2 * u) * np.abs(out) + 1e-30
    return tol, delta + count * u + 8 * u


class Scene:
    """Sequences over random pages: `lens` tokens each, pages in random order,
    rows behind a sequence's last one filled with anything (NaN scales among
    it).  `cold`: that many of the ids lie in the cold tier."""

    def __init__(self, hga, dtype="bf16", d=64, kv=2, ratio=2, lens=(130,), seed=0, cold=0, spare=2,
                 max_pages=None, layers=1, layer=0, first=1, last=0, prev=1, topk=2, base=1e4):
        rng = np.random.default_rng(seed)
        self.hga, self.dtype, self.d, self.kv, self.hq, self.rng = hga, dtype, d, kv, kv * ratio, rng
        self.first, self.window, self.topk, self.base = first, max(last, prev), topk, base
        self.plan = hga.Plan(batch=1, n_q_heads=self.hq, n_kv_heads=kv, head_dim=d, keep_first=first,
                             keep_last=last, force_prev=prev, topk_chunks=topk, topk_groups=4,
                             dtype=hga.F32 if dtype == "f32" else hga.BF16, rope_base=base)
        self.lens, self.layer = list(lens), layer
        need = [-(-n // PAGE) for n in lens]
        self.max_pages = max_pages or max(need + [1])
        n = sum(need) + spare
        self.n_ids, hb = n, head_bytes(d)
        b = rng.integers(0, 256, (n, kv, hb), dtype=np.uint8)
        kc, ks, vc, vs = addresses(d)
        b[..., 64 * d:] = rng.integers(122, 129, (n, kv, hb - 64 * d))
        ids = rng.permutation(n)
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        at = 0
        for s, x in enumerate(need):
            self.table[s, :x] = ids[at:at + x]
            at += x
            if lens[s] % PAGE:
                b[self.table[s, x - 1]][:, ks[lens[s] % PAGE:]] = 255
                b[self.table[s, x - 1]][:, vs[lens[s] % PAGE:]] = 255
        self.bytes = b
        self.sums = rng.standard_normal((n, kv, d)).astype(np.float32)
        hot = n - cold
        pages = torch.full((layers, hot, kv, hb), 255, dtype=torch.uint8)
        pages[layer] = torch.from_numpy(b[:hot])
        sums = torch.full((layers, n, kv, d), float("nan"))
        sums[layer] = torch.from_numpy(self.sums)
        cold_t = None
        if cold:
            cold_t = torch.full((layers, cold, kv, hb), 255, dtype=torch.uint8).pin_memory()
            cold_t[layer] = torch.from_numpy(b[hot:])
        self.pool = hga.Pool(self.plan, pages=pages.cuda(), page_sum=sums.cuda(), cold=cold_t)

    def k_v(self):
        return page_values(self.bytes, self.d)

    def stored(self):
        """The layer's page bytes now, hot then cold."""
        torch.cuda.synchronize()
        b = self.pool.pages[self.layer].cpu().numpy()
        if self.pool.cold is not None:
            b = np.concatenate((b, self.pool.cold[self.layer].numpy()))
        return b

    def batch(self, seq, pos):
        i32 = lambda x: torch.tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
        self.seq, self.pos = np.asarray(seq, np.int64), np.asarray(pos, np.int64)
        return self.hga.TokenBatch(i32(seq).reshape(-1), i32(pos).reshape(-1), i32(self.table))

    def random(self, *shape, scale=1.0):
        x = torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32) * scale)
        return x.to(DT[self.dtype]).cuda()

    def route(self, batch, q, extra=0, stream=None):
        hga = self.hga
        n = hga.hga_token_list_size(self.plan) + extra
        out = torch.full((batch.n_tokens, self.kv, n), -7, dtype=torch.int32, device="cuda")
        nb = hga.hga_route_tokens_workspace(self.plan, batch)
        ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
        hga.hga_route_tokens(self.plan, self.pool, self.layer, batch, q, out, workspace=ws, stream=stream)
        return out

    def attend(self, batch, q, lists=None, workspace=True, stream=None):
        hga = self.hga
        out = torch.full((batch.n_tokens, self.hq, self.d), float("nan"), dtype=DT[self.dtype], device="cuda")
        lse = torch.full((batch.n_tokens, self.hq), float("nan"), device="cuda")
        ws = None
        if workspace:
            nb = hga.hga_attend_tokens_workspace(self.plan, batch, lists) if workspace is True else workspace
            ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda") if nb else None
        hga.hga_attend_tokens(self.plan, self.pool, self.layer, batch, q, out, lse=lse, chunk_list=lists,
                              workspace=ws, stream=stream)
        return out, lse

    def check_attend(self, q, got, lists=None, tokens=slice(None)):
        """Of the given tokens of a call (all)."""
        out, lse = got
        k, v = self.k_v()
        ln = None if lists is None else lists.cpu().numpy()[tokens]
        ref, rlse, mag, reach, count = attend(f64(q)[tokens], k, v, self.table, self.seq[tokens], self.pos[tokens],
                                              self.kv, ln, self.n_ids)
        tol, ltol = attend_tolerance(self.dtype, self.d, ref, mag, reach, count)
        o, l = f64(out)[tokens], f64(lse)[tokens]
        none = count == 0
        assert (o[none] == 0).all() and (l[none] == -np.inf).all()
        assert np.isfinite(o).all() and np.isfinite(l[~none]).all()
        err, lerr = np.abs(o - ref), np.abs(l[~none] - rlse[~none])
        assert (err <= tol).all(), float((err / tol).max())
        assert (lerr <= ltol[~none]).all(), float((lerr / ltol[~none]).max())
