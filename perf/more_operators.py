"""More of the paged 4-bit cache's operators as they are timed: attention of a
batch whose sequences share leading pages, the attention weight that pages
accumulate, and the choice of the pages to evict by it.

Each case is one call of a serving loop over sequences that are rows of a page
table.  With ``own`` false the operators run in their plain form (elementary
torch operations in 32 or 64 bits), with ``own`` true through
``paper_2606_30709_amd.hga``.

A page holds 64 consecutive tokens of one sequence for every KV head.  One KV
head's part of a page, in bytes (d = head_dim):

* 64 * d/2    key codes, row by row (dimension 2i in the low half of byte i);
* 64 * d/2    value codes ``[16 quads of rows][16][4 rows][d/16 dimensions]``;
* 64 * d/32   key scales ``[row % 16][d/32 blocks][row / 16]``;
* 64 * d/32   value scales ``[(row / 4) % 4][d/32 blocks][row / 16][row % 4]``.

A code is a sign and a magnitude of {0, 0.5, 1, 1.5, 2, 3, 4, 6}; 32 dimensions
of a row share a power-of-two scale, stored as its exponent + 127.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 64
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases ---

def _named(name, c):
    return dict(name=name, **c) if name else c


def _shared(name, dtype, kv, ratio, d, groups, members, prefix, tail, new=1, alone=0):
    """`groups` groups of sequences, members[0] to members[1] in each, which
    share their first prefix[0] to prefix[1] pages and go on by themselves for
    tail[0] to tail[1] tokens, the last min(new, tail) of them being this
    call's; and `alone` sequences that share nothing."""
    return _named(name, dict(do="shared", dtype=dtype, kv=kv, ratio=ratio, d=d, groups=groups,
                             members_lo=members[0], members_hi=members[1], prefix_lo=prefix[0],
                             prefix_hi=prefix[1], tail_lo=tail[0], tail_hi=tail[1], new=new,
                             alone=alone))


def _weigh(name, dtype, kv, ratio, d, seqs, lo, hi, new=1, first=1, last=0, kc=8, sparse=False):
    """seqs sequences whose lengths (this call's tokens included) spread over
    [lo, hi], the last min(new, length) tokens of each being this call's."""
    return _named(name, dict(do="weigh", dtype=dtype, kv=kv, ratio=ratio, d=d, seqs=seqs, lo=lo,
                             hi=hi, new=new, first=first, last=last, kc=kc, sparse=sparse))


def _choose(name, kv, seqs, lo, hi, keep, first=1, last=0):
    """seqs sequences of lo to hi pages, of which each keeps the share `keep`."""
    return _named(name, dict(do="choose", dtype="bf16", kv=kv, ratio=1, d=64, seqs=seqs, lo=lo,
                             hi=hi, keep=keep, first=first, last=last))


def listed():
    return [
        # three short answers after one 640-token prompt: the smallest call
        _shared("shared_few", "f32", 2, 3, 64, 1, (3, 3), (10, 10), (1, 70)),
        # a decode step of 64 samples of one 16K prompt
        _shared("shared_samples", "bf16", 4, 8, 128, 1, (64, 64), (256, 256), (1, 2048)),
        # a decode step of many prompts, a few samples each, and of some that share nothing
        _shared("shared_groups", "bf16", 8, 1, 64, 12, (2, 16), (20, 128), (1, 600), alone=8),
        # four drafted tokens of 16 sequences after an 8K prompt, fp32
        _shared("shared_drafts", "f32", 3, 4, 128, 1, (16, 16), (128, 128), (4, 300), new=4),
        # sixteen questions of 128 tokens about one 16K document (the largest)
        _shared("shared_questions", "bf16", 4, 8, 128, 1, (16, 16), (256, 256), (128, 128),
                new=128),
        # one token over a short history, fp32
        _weigh("weigh_one", "f32", 2, 3, 64, 1, 700, 700),
        # a decode step of 32 sequences over their whole histories
        _weigh("weigh_decode", "bf16", 4, 8, 128, 32, 1000, 32768),
        # a decode step of 64 sequences over routed pages
        _weigh("weigh_routed", "bf16", 4, 8, 128, 64, 1000, 65536, first=2, last=8, kc=20,
               sparse=True),
        # the last 32 tokens of ragged prompts as observers of the whole prompt, fp32
        _weigh("weigh_window", "f32", 12, 1, 64, 6, 1021, 8192, new=32),
        # one sequence of 128K tokens cut to a quarter
        _choose("choose_one", 4, 1, 2048, 2048, 0.25, first=2, last=8),
        # a batch that has to shrink by a tenth
        _choose("choose_batch", 8, 64, 100, 2048, 0.9),
        # eight sequences of up to a million tokens, by half
        _choose("choose_long", 8, 8, 2000, 16384, 0.5, first=2, last=8),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def span(lo, hi):
        b = log_int(lo, hi)
        return log_int(lo, b), b

    limits = {}
    for c in listed():
        limits[c["do"]] = max(limits.get(c["do"], 0.0), _cost(c))
    while True:
        do = rng.choice(["shared", "shared", "weigh", "weigh", "choose"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([64, 128])
        kv = rng.choice([1, 2, 3, 4, 5, 8, 12])
        ratio = rng.choice([1, 2, 3, 4, 6, 8])
        first, last = rng.randint(0, 2), rng.choice([0, 0, 1, 2, 8])
        if do == "choose":
            lo, hi = span(1, 16384)
            c = _choose("", kv, log_int(1, 64), lo, hi, round(rng.uniform(0.05, 1.0), 3),
                        first=first, last=last)
        elif do == "shared":
            # a decode step, a draft or a prompt after the shared pages
            new = rng.choice([1, 1, log_int(2, 8), log_int(2, 256)])
            groups = log_int(1, 24)
            c = _shared("", dtype, kv, ratio, d, groups, span(1, 64), span(1, 512),
                        span(1, 2048), new, rng.choice([0, 0, log_int(1, 16)]))
        else:
            lo, hi = span(1, 32768)
            new = rng.choice([1, 1, log_int(2, 32), log_int(2, 512)])
            c = _weigh("", dtype, kv, ratio, d, log_int(1, 64), lo, hi, new, first=first,
                       last=last, kc=log_int(2, 30), sparse=rng.random() < 0.4)
        if _cost(c) <= limits[do] and (do == "choose" or _pool_bytes(c) <= 1.5e9):
            return c


def _cost(c):
    """What a case costs at most: bytes, and arithmetic at about 50 a byte."""
    w = work(c)
    return max(w["bytes"], w["flops"] / 50.0)


def _spread(lo, hi, i, n):
    return lo + (hi - lo) * i // max(n - 1, 1)


def _lens(c):
    """(group or -1, shared pages, length, new tokens) of every sequence."""
    if c["do"] == "weigh":
        lens = [_spread(c["lo"], c["hi"], i, c["seqs"]) for i in range(c["seqs"])]
        return [(-1, 0, x, min(c["new"], x)) for x in lens]
    where = []
    for g in range(c["groups"]):
        # the groups of the longest prompts are the smallest
        pages = _spread(c["prefix_hi"], c["prefix_lo"], g, c["groups"])
        where += [(g, pages)] * _spread(c["members_lo"], c["members_hi"], g, c["groups"])
    where += [(-1, 0)] * c["alone"]
    out = []
    for i, (g, pages) in enumerate(where):
        # lengths of neighbours differ: sequences of one group are short and long
        tail = _spread(c["tail_lo"], c["tail_hi"], i * 7 % len(where), len(where))
        out.append((g, pages, pages * PAGE + tail, min(c["new"], tail)))
    return out


def _window(c):
    return max(c["last"], 1)


def _list_size(c):
    return c["first"] + _window(c) + c["kc"] + 1


def _head_bytes(d):
    return PAGE * (d + d // 16)


def _n_pages(c):
    """Pages of the pool that hold rows: shared ones once."""
    lens = _lens(c)
    return sum(-(-x // PAGE) - p for _, p, x, _ in lens) + sum({g: p for g, p, _, _ in lens}.values())


def _pool_bytes(c):
    return (_n_pages(c) + 3) * c["kv"] * _head_bytes(c["d"])


def _page_counts(c):
    return [_spread(c["lo"], c["hi"], i, c["seqs"]) for i in range(c["seqs"])]


def _visible(c, own_chunk):
    """Chunks in the list of a token in chunk own_chunk."""
    mid = max(0, own_chunk - _window(c) - c["first"])
    return own_chunk + 1 - mid + min(mid, c["kc"])


def work(c):
    kv, d, do = c["kv"], c["d"], c["do"]
    hq, elt = kv * c["ratio"], 2 if c["dtype"] == "bf16" else 4
    if do == "choose":
        n = float(sum(_page_counts(c)))
        gone = sum(x - math.ceil(c["keep"] * x) for x in _page_counts(c))
        # weights and table words in, the list out
        return {"bytes": n * (4 * kv + 4) + 4.0 * gone + 8.0 * c["seqs"], "flops": n * kv}
    row = d // 2 + d // 32
    byts = flops = 0.0
    seen = {}
    for g, p, x, new in _lens(c):
        where = range(x - new, x)
        if do == "shared":
            rows = x - p * PAGE + (0 if g in seen else p * PAGE)   # a group's pages once
            if g >= 0:
                seen[g] = p
            byts += kv * 2.0 * rows * row + new * hq * (2.0 * d * elt + 4) + 8.0 * new
            flops += 4.0 * hq * d * sum(t + 1 for t in where)
        else:
            keys = [(_visible(c, t // PAGE) - 1) * PAGE + t % PAGE + 1 if c["sparse"] else t + 1
                    for t in where]
            rows = min(x, sum(keys)) if c["sparse"] else x
            # keys, queries and lse in; weights in and out
            byts += kv * (1.0 * rows * row + 8.0 * (-(-x // PAGE))) + new * hq * (d * elt + 4.0)
            if c["sparse"]:
                byts += 4.0 * new * kv * _list_size(c)
            flops += 2.0 * hq * d * sum(keys)
    return {"bytes": byts, "flops": flops}


# ----------------------------------------------------------------- format ---

def _encode(x):
    """fp32 [..., d] -> codes uint8 [..., d], scale bytes uint8 [..., d/32], of
    finite values well inside fp32's range."""
    b = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bits = b.abs().amax(-1).view(torch.int32)
    e = ((bits >> 23) - 2 + ((bits & 0x7FFFFF) > 0x400000).int()).clamp(2, 253)
    y = b.abs() * torch.exp2(127.0 - e.double()).float()[..., None]
    code = ((y > 0.25).int() + (y >= 0.75).int() + (y > 1.25).int() + (y >= 1.75).int() +
            (y > 2.5).int() + (y >= 3.5).int() + (y > 5.0).int())
    code = torch.where(torch.signbit(b), code + 8, code)
    return code.to(torch.uint8).reshape(x.shape), e.to(torch.uint8)


def _decode(codes, scales):
    """codes [..., d], scale bytes [..., d/32] -> fp32 values."""
    i = torch.arange(16, device=codes.device)
    mag = torch.where(i % 8 < 4, (i % 8) * 0.5, (2 + i % 2) * torch.exp2((i % 8) // 2 - 2.0))
    mag = torch.where(i < 8, mag, -mag)
    sc = torch.exp2(torch.arange(256, device=codes.device).double() - 127).float()
    v = mag[codes.int()].reshape(*scales.shape, 32) * sc[scales.int()][..., None]
    return v.reshape(codes.shape)


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _pair(codes):
    c = codes.unflatten(-1, (-1, 2))
    return c[..., 0] | (c[..., 1] << 4)


def _parts(pages, d):
    """Views of a [..., head_bytes] page tensor: key codes, value codes, key
    scales, value scales."""
    n, nb = PAGE * d // 2, d // 32
    k = pages[..., :n].unflatten(-1, (PAGE, d // 2))
    v = pages[..., n:2 * n].unflatten(-1, (16, 16, 4, d // 32))
    ks = pages[..., 2 * n:2 * n + PAGE * nb].unflatten(-1, (16, nb, 4))
    vs = pages[..., 2 * n + PAGE * nb:].unflatten(-1, (4, nb, 4, 4))
    return k, v, ks, vs


def _unpack_k(pages, d):
    k, _, ks, _ = _parts(pages, d)
    return _decode(_nibbles(k), ks.movedim(-1, -3).flatten(-3, -2))


def _unpack_v(pages, d):
    _, v, _, vs = _parts(pages, d)
    codes = _nibbles(v).movedim(-2, -3)                       # [quad, row % 4, 16, d/16]
    scales = vs.movedim(-3, -1).movedim(-4, -3)               # [t, g, row % 4, block]
    return _decode(codes.flatten(-2).flatten(-3, -2), scales.flatten(-4, -2))


def _fill_pages(part, k, v):
    """Whole pages part [n, kv, bytes] from k, v [n, kv, 64, d]."""
    d = k.shape[-1]
    kd, vd, ks, vs = _parts(part, d)
    off = torch.arange(PAGE, device=k.device)
    kc, kscale = _encode(k)
    vc, vscale = _encode(v)
    kd[:] = _pair(kc)
    ks[:, :, off % 16, :, off // 16] = kscale.movedim(2, 0)
    vd[:, :, off // 4, :, off % 4] = _pair(vc).unflatten(-1, (16, d // 32)).movedim(2, 0)
    vs[:, :, (off % 16) // 4, :, off // 16, off % 4] = vscale.movedim(2, 0)


# ----------------------------------------------------------------- inputs ---

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    st = _prepare_inputs(case, seed)
    if own:
        _prepare_own(st)
    return st


def _prepare_inputs(case, seed):
    c = case
    g = _generator(seed)
    return _prepare_choose(c, g) if c["do"] == "choose" else _prepare_cache(c, g)


def _prepare_choose(c, g):
    dev, counts = "cuda", _page_counts(c)
    S, n = len(counts), max(counts)
    # pages of any order; one in fifty has been dropped before
    table = torch.stack([torch.randperm(S * n, device=dev, generator=g)[:n] for _ in counts]).int()
    count = torch.tensor(counts, device=dev)
    gone = torch.rand(S, n, device=dev, generator=g) < 0.02
    table[gone | (torch.arange(n, device=dev) >= count[:, None])] = -1
    # lengths end anywhere in the last page; attention weights spread over
    # decades, and some pages were never looked at: exact zeros, which tie
    length = count * PAGE - torch.randint(0, PAGE, (S,), device=dev, generator=g)
    w = torch.exp(3.0 * torch.randn(S, c["kv"], n, device=dev, generator=g))
    w *= (torch.rand(S, 1, n, device=dev, generator=g) >= 0.1)
    keep = torch.tensor([math.ceil(c["keep"] * x) for x in counts], device=dev)
    most = max(1, max(x - math.ceil(c["keep"] * x) for x in counts))
    return dict(case=c, table=table, length=length.int(), weights=w, budget=keep.int(),
                n_pages=S * n, evicted=torch.empty(S, most, dtype=torch.int32, device=dev))


def _prepare_cache(c, g):
    d, kv, dev, dt = c["d"], c["kv"], "cuda", DT[c["dtype"]]
    lens, hq = _lens(c), kv * c["ratio"]
    n_pages = _n_pages(c) + 3

    # the pool: keys with a direction of their own per page (so that pages get
    # different shares of the attention, as passages of a text do), plain values
    pages = torch.empty(1, n_pages, kv, _head_bytes(d), dtype=torch.uint8, device=dev)
    step = max(1, (1 << 24) // (kv * PAGE * d))
    for a in range(0, n_pages, step):
        n = min(step, n_pages - a)
        k = torch.randn(n, kv, PAGE, d, device=dev, generator=g)
        k += 1.5 * torch.randn(n, kv, 1, d, device=dev, generator=g)
        _fill_pages(pages[0, a:a + n], k, torch.randn(n, kv, PAGE, d, device=dev, generator=g))

    # sequences stand in any order in the table, their pages in any order in the pool
    rows = torch.randperm(len(lens), device=dev, generator=g).tolist()
    ids = torch.randperm(n_pages, device=dev, generator=g).tolist()
    max_pages = max(-(-x // PAGE) for _, _, x, _ in lens)
    table = np.full((len(lens), max_pages), -1, np.int32)
    prefix = {}
    for s, i in enumerate(rows):
        grp, p, x, _ = lens[i]
        if grp not in prefix:
            prefix[grp] = [ids.pop() for _ in range(p)]
        table[s, :p] = prefix[grp]
        table[s, p:-(-x // PAGE)] = [ids.pop() for _ in range(-(-x // PAGE) - p)]
    seq = np.concatenate([np.full(lens[i][3], s, np.int32) for s, i in enumerate(rows)])
    pos = np.concatenate([np.arange(lens[i][2] - lens[i][3], lens[i][2], dtype=np.int32)
                          for i in rows])
    T = len(seq)
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(dev)  # noqa: E731
    st = dict(case=c, rows=rows, pages=pages, table=up(table), seq=up(seq), pos=up(pos),
              q=torch.randn(T, hq, d, device=dev, generator=g).to(dt))
    st["lse"] = torch.empty(T, hq, device=dev)
    if c["do"] == "shared":
        G = c["groups"]
        of = np.array([lens[i][0] % (G + 1) for i in rows])[seq]      # the last for those alone
        order = np.argsort(of, kind="stable")
        st.update(order=up(order.astype(np.int32)), out=torch.empty_like(st["q"]),
                  begin=up(np.searchsorted(of[order], np.arange(G + 1)).astype(np.int32)),
                  shared=up(np.array([{g: p for g, p, _, _ in lens}[g] for g in range(G)],
                                     np.int32)))
        return st
    if c["sparse"]:
        # visible chunks, random middle ones, the token's own, ascending
        o, W, F, kc = (st["pos"] // PAGE).long(), _window(c), c["first"], c["kc"]
        st["list"] = torch.full((T, kv, _list_size(c)), -1, dtype=torch.int32, device=dev)
        col = torch.arange(max_pages, device=dev)
        for a in range(0, T, 256):
            ob = o[a:a + 256, None, None]
            key = torch.rand(len(ob), kv, max_pages, device=dev, generator=g)
            key = torch.where((col >= F) & (col < ob - W), key, torch.full_like(key, -1.0))
            keep = (col <= ob) & ((col < F) | (col >= ob - W))
            keep = keep.expand(len(ob), kv, max_pages).clone()
            top = key.topk(min(kc, max_pages), -1)
            keep.scatter_(-1, top.indices, keep.gather(-1, top.indices) | (top.values >= 0))
            rank = keep.cumsum(-1) - 1
            t, h, ci = keep.nonzero(as_tuple=True)
            st["list"][a + t, h, rank[t, h, ci]] = ci.int()
    # what a few earlier tokens left (as much as this call's: neither hides the
    # other), and the lse that the step's attention gave
    st["prev"] = torch.rand(len(lens), kv, max_pages, device=dev, generator=g)
    st["prev"] *= 2.0 * c["ratio"] / max_pages
    st["weights"] = torch.empty_like(st["prev"])
    for a, b, _, score in _scores(st):
        st["lse"][a:b] = torch.logsumexp(score, -1).flatten(1)
    return st


def _prepare_own(st):
    from paper_2606_30709_amd import hga
    c = st["case"]
    plan = hga.Plan(batch=1, n_q_heads=c["kv"] * c["ratio"], n_kv_heads=c["kv"], head_dim=c["d"],
                    keep_first=c.get("first", 1), keep_last=c.get("last", 0), force_prev=1,
                    topk_chunks=c.get("kc", 8), topk_groups=4,
                    dtype=hga.F32 if c["dtype"] == "f32" else hga.BF16, rope_base=1e4)
    st["plan"] = plan
    if c["do"] == "choose":
        nbytes = hga.hga_choose_evictions_workspace(plan, st["table"])
    else:
        st["pool"] = hga.Pool(plan, pages=st["pages"])
        st["batch"] = hga.TokenBatch(st["seq"], st["pos"], st["table"])
    if c["do"] == "shared":
        # (with the longest shared and unshared parts, as a cache's bookkeeping knows them)
        st["prefixes"] = hga.Prefixes(st["order"], st["begin"], st["shared"],
                                      max(p for _, p, _, _ in _lens(c)),
                                      max(-(-x // PAGE) - p for _, p, x, _ in _lens(c)))
        nbytes = hga.hga_attend_shared_workspace(plan, st["batch"], st["prefixes"])
    elif c["do"] == "weigh":
        nbytes = hga.hga_weigh_pages_workspace(plan, st["batch"], st.get("list"))
    st["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


# -------------------------------------------------------------- one pass ---

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2606_30709_amd import hga
    do = st["case"]["do"]
    if do == "choose":
        hga.hga_choose_evictions(st["plan"], st["table"], st["n_pages"], st["length"],
                                 st["weights"], st["budget"], st["evicted"],
                                 workspace=st["workspace"])
        return st["evicted"]
    if do == "shared":
        hga.hga_attend_shared(st["plan"], st["pool"], 0, st["batch"], st["prefixes"], st["q"],
                              st["out"], lse=st["lse"], workspace=st["workspace"])
        return st["out"], st["lse"]
    hga.hga_weigh_pages(st["plan"], st["pool"], 0, st["batch"], st["q"], st["lse"], st["weights"],
                        prev=st["prev"], chunk_list=st.get("list"), workspace=st["workspace"])
    return st["weights"]


def _run_plain(st):
    return {"shared": _plain_shared, "weigh": _plain_weigh, "choose": _plain_choose}[
        st["case"]["do"]](st)


def _runs(st):
    """(table row, its entry of _lens, tokens [a, b)) in the batch's order."""
    lens, a = _lens(st["case"]), 0
    for s, i in enumerate(st["rows"]):
        yield s, lens[i], a, a + lens[i][3]
        a += lens[i][3]


def _plain_shared(st):
    """Running maxima m, sums l and results o: those over a group's pages for
    all of its tokens at once, then each sequence's own are joined to them."""
    c = st["case"]
    d, kv, r = c["d"], c["kv"], c["ratio"]
    pages, table, dev = st["pages"][0], st["table"].long(), st["q"].device
    T = len(st["pos"])
    q = st["q"].float().unflatten(1, (kv, r)).transpose(0, 1).contiguous()     # [kv, T, r, d]
    o = torch.zeros(kv, T, r, d, device=dev)
    m = torch.full((kv, T, r), -math.inf, device=dev)
    l = torch.zeros(kv, T, r, device=dev)
    of = {}
    for s, (g, p, _, _), a, b in _runs(st):
        of.setdefault(g, (s, p, []))[2].extend(range(a, b))

    def add(ts, ids, first):
        """Pages `ids`, whose rows are positions from `first` on, for tokens ts."""
        n = len(ids) * PAGE
        block = pages[ids].transpose(0, 1)                                     # [kv, n, bytes]
        k, v = (f(block, d).flatten(1, 2).contiguous() for f in (_unpack_k, _unpack_v))
        kt = k.transpose(-1, -2).contiguous()
        step = max(1, (1 << 28) // (kv * r * n))
        for a in range(0, len(ts), step):
            t = ts[a:a + step]
            x = torch.matmul(q[:, t].flatten(1, 2), kt).unflatten(1, (-1, r)) / math.sqrt(d)
            see = first + torch.arange(n, device=dev) <= st["pos"][t].long()[:, None, None]
            x = torch.where(see, x, torch.full_like(x, -math.inf))
            top = torch.maximum(m[:, t], x.amax(-1))
            w = (x - top[..., None]).exp()
            f = (m[:, t] - top).exp()
            l[:, t] = l[:, t] * f + w.sum(-1)
            o[:, t] = o[:, t] * f[..., None] + \
                torch.matmul(w.flatten(1, 2), v).unflatten(1, (-1, r))
            m[:, t] = top

    for g, (s, p, ts) in of.items():
        if g >= 0:
            add(torch.tensor(ts, device=dev), table[s, :p], 0)
    for s, (_, p, x, _), a, b in _runs(st):
        add(torch.arange(a, b, device=dev), table[s, p:-(-x // PAGE)], p * PAGE)
    out = (o / l[..., None]).transpose(0, 1).flatten(1, 2)
    return out.to(st["q"].dtype), (m + l.log()).transpose(0, 1).flatten(1, 2)


def _scores(st):
    """Scores in fp32, a sequence's tokens (or, with lists, any tokens) at a
    time: tokens [a, b), chunks [kv, n] (or [b - a, kv, n]) and s [b - a, kv, r,
    rows of the chunks]; a row that a token does not see has a score of -inf."""
    c = st["case"]
    d, kv, r = c["d"], c["kv"], c["ratio"]
    pages, table, dev = st["pages"][0], st["table"].long(), st["q"].device
    row, heads = torch.arange(PAGE, device=dev), torch.arange(kv, device=dev)[:, None]
    masked = lambda see, s: torch.where(see, s, torch.full_like(s, -math.inf))  # noqa: E731
    if c["sparse"]:
        step = max(1, (1 << 25) // (kv * st["list"].shape[-1] * PAGE * d))
        for a in range(0, len(st["pos"]), step):
            ci, pos = st["list"][a:a + step].long(), st["pos"][a:a + step].long()
            seq = st["seq"][a:a + step].long()[:, None, None]
            k = _unpack_k(pages[table[seq, ci.clamp(min=0)], heads], d).flatten(2, 3)
            at = (ci[..., None] * PAGE + row).flatten(2)
            see = (ci >= 0).repeat_interleave(PAGE, -1) & (at <= pos[:, None, None])
            q = st["q"][a:a + step].float().unflatten(1, (kv, r))
            s = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(d)
            yield a, a + len(ci), ci, masked(see[:, :, None], s)
        return
    for s_id, (_, _, x, _), start, end in _runs(st):
        n = -(-x // PAGE)
        kt = _unpack_k(pages[table[s_id, :n]], d).transpose(0, 1).flatten(1, 2)
        kt = kt.transpose(-1, -2).contiguous()                                 # [kv, d, rows]
        step = max(1, (1 << 28) // (kv * r * n * PAGE))
        for a in range(start, end, step):
            b = min(a + step, end)
            q = st["q"][a:b].float().unflatten(1, (kv, r)).transpose(0, 1).flatten(1, 2)
            s = torch.matmul(q, kt).unflatten(1, (b - a, r)).transpose(0, 1) / math.sqrt(d)
            see = torch.arange(n * PAGE, device=dev) <= st["pos"][a:b].long()[:, None, None, None]
            yield a, b, torch.arange(n, device=dev).expand(kv, n), masked(see, s)


def _plain_weigh(st):
    c = st["case"]
    w = st["weights"].copy_(st["prev"])
    heads = torch.arange(c["kv"], device=w.device)[:, None]
    for a, b, chunks, s in _scores(st):
        p = (s - st["lse"][a:b].unflatten(1, (c["kv"], c["ratio"]))[..., None]).exp()
        total = p.unflatten(-1, (-1, PAGE)).sum(-1).sum(2)                     # [t, kv, n]
        if chunks.dim() == 2:
            w[st["seq"][a].long(), :, :chunks.shape[1]] += total.sum(0)
        else:
            # places behind a list's end add nothing to chunk 0
            seq = st["seq"][a:b].long()[:, None, None].expand_as(chunks)
            w.index_put_((seq, heads.expand_as(chunks), chunks.clamp(min=0)), total, accumulate=True)
    return w


def _plain_choose(st):
    c = st["case"]
    out = st["evicted"].fill_(-1)
    S, n = st["table"].shape
    col = torch.arange(n, device=out.device)
    last = ((st["length"] - 1) // PAGE).long()[:, None]
    here = (st["table"] >= 0) & (st["table"] < st["n_pages"]) & (col <= last)
    may = here & (col >= c["first"]) & (col < last - _window(c))
    # sums in 64 bits: those next to the border decide which page goes
    score = st["weights"].double().sum(1)
    score = torch.where(may, score, torch.full_like(score, math.inf))
    # stable: of equal sums the lowest chunk first
    rank = score.sort(dim=-1, stable=True).indices
    gone = torch.minimum(here.sum(-1) - st["budget"], may.sum(-1)).clamp(0, out.shape[1])
    pick = torch.where(col < gone[:, None], rank, n)[:, :out.shape[1]].sort(-1).values
    out[:, :pick.shape[1]] = torch.where(pick < n, pick, -1).int()
    return out


# ----------------------------------------------------------- definition ---

def _element_values(block, d, which):
    """fp64 values [..., 64, d] of a page's keys or values, each element looked
    up by its own byte address."""
    o = np.arange(PAGE)[:, None]
    j = np.arange(d)[None, :]
    half = PAGE * d // 2
    if which == "k":
        at = o * (d // 2) + j // 2
        sc = 2 * half + ((o % 16) * (d // 32) + j // 32) * 4 + o // 16
    else:
        dl = d // 16
        at = half + ((o // 4) * 16 + j // dl) * (2 * dl) + (o % 4) * (dl // 2) + (j % dl) // 2
        sc = 2 * half + PAGE * (d // 32) + \
            (((o // 4) % 4 * (d // 32) + j // 32) * 4 + o // 16) * 4 + o % 4
    dev = block.device
    at, sc, shift = (torch.from_numpy(np.broadcast_to(x, (PAGE, d)).copy()).to(dev)
                     for x in (at, sc, 4 * (j % 2)))
    code = (block[..., at].long() >> shift) & 15
    exp = block[..., sc].long()
    # magnitude of a code with exponent field x and one fraction bit f:
    # f / 2 for x = 0, (1 + f / 2) 2^(x - 1) otherwise
    x, f = (code >> 1) & 3, (code & 1).double()
    mag = torch.where(x == 0, f / 2, (1 + f / 2) * 2.0 ** (x - 1).double())
    return mag * torch.where(code >= 8, -1.0, 1.0) * 2.0 ** (exp - 127).double()


def exact(case, seed):
    c = case
    st = _prepare_inputs(case, seed)
    table = st["table"].cpu().numpy()
    if c["do"] == "choose":
        out = np.full(tuple(st["evicted"].shape), -1, np.int32)
        w, length = st["weights"].double().cpu().numpy(), st["length"].tolist()
        for s, budget in enumerate(st["budget"].tolist()):
            last = (length[s] - 1) // PAGE
            here = [x for x in range(last + 1) if 0 <= table[s, x] < st["n_pages"]]
            may = np.array([x for x in here if c["first"] <= x < last - _window(c)], np.int64)
            gone = min(max(len(here) - budget, 0), len(may), out.shape[1])
            if gone:
                total = sum(w[s, h, may] for h in range(c["kv"]))
                pick = may[np.lexsort((may, total))[:gone]]
                out[s, :gone] = np.sort(pick)
        return torch.from_numpy(out)
    d, kv, r = c["d"], c["kv"], c["ratio"]
    seq = st["seq"].tolist()
    T, sparse = len(seq), c["do"] == "weigh" and c["sparse"]
    if c["do"] == "shared":
        out = torch.empty(T, kv * r, d, dtype=torch.float64, device="cuda")
        lse = torch.empty(T, kv * r, dtype=torch.float64, device="cuda")
    else:
        weights = st["prev"].double()
    for s in sorted(set(seq)):
        n = int((table[s] >= 0).sum())
        toks = [t for t in range(T) if seq[t] == s]
        for h in range(kv):
            block = st["pages"][0, st["table"][s, :n].long(), h]
            k = _element_values(block, d, "k").flatten(0, 1)
            v = _element_values(block, d, "v").flatten(0, 1) if c["do"] == "shared" else None
            for a in range(0, len(toks), 64):
                ts = torch.tensor(toks[a:a + 64], device="cuda")
                heads = slice(h * r, (h + 1) * r)
                q, x = st["q"][ts, heads].double(), st["pos"][ts].long()
                see = torch.arange(n * PAGE, device="cuda") <= x[:, None]
                if sparse:
                    opened = torch.zeros(len(ts), n + 1, dtype=torch.bool, device="cuda")
                    ids = st["list"][ts, h].long()
                    opened.scatter_(1, torch.where(ids < 0, n, ids), True)
                    see &= opened[:, :n].repeat_interleave(PAGE, 1)
                sc = torch.tensordot(q, k, dims=([2], [1])) / math.sqrt(d)
                sc = sc.masked_fill(~see[:, None], -math.inf)
                if c["do"] == "shared":
                    norm = torch.logsumexp(sc, -1)
                    w = torch.exp(sc - norm[..., None])
                    out[ts, heads] = torch.tensordot(w, v, dims=([2], [0]))
                    lse[ts, heads] = norm
                else:
                    w = torch.exp(sc - st["lse"][ts, heads, None].double())
                    weights[s, h, :n] += w.unflatten(-1, (n, PAGE)).sum((0, 1, 3))
    return (out, lse) if c["do"] == "shared" else weights
