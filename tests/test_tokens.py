"""Single tokens over the paged 4-bit cache against 64-bit definitions
(tokens_util): what is stored, which pages are listed, what attention gives."""

from __future__ import annotations

import numpy as np
import pytest
import torch

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


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


def _same(a, b):
    return all(torch.equal(_bits(x), _bits(y)) for x, y in zip(a, b))


SHAPES = [("bf16", 128, 4, 8), ("f32", 128, 1, 16), ("bf16", 64, 3, 3), ("f32", 64, 2, 1), ("bf16", 64, 1, 16),
          ("bf16", 128, 5, 2), ("f32", 128, 2, 5), ("f32", 128, 2, 4), ("f32", 64, 3, 3)]


# ------------------------------------------------------------- the store ---

def _special(rng, T, kv, d):
    """Rows with what a quantiser meets: ties, a large dynamic range, zeros,
    subnormals, the largest floats, infinities, NaN."""
    x = rng.standard_normal((T, kv, d)).astype(np.float32)
    x[0] = np.resize([6, 5, 3.5, 2.5, 1.75, 1.25, .75, .25, -.25, -5, 0, -0.0, 4, 2, 6, 1], d)
    x[1 % T, :, :32] = 0
    x[2 % T, :, :32] *= 4e-39
    x[3 % T, :, :32] = np.resize([3.3895e38, -3.38e38, 2.6e38, -2.9e38, 1e38, 3e37, 1], 32)
    x[4 % T, :, 5] = np.inf
    x[5 % T, :, 40] = np.nan
    x[6 % T, :, 7] *= 1e4
    x[7 % T, :, 33:] = 2.0 ** -126
    x[8 % T] *= np.exp2(rng.integers(-120, 120, (kv, d // 32))).repeat(32, -1).astype(np.float32)
    return x


@pytest.mark.parametrize("dtype,d,kv,ratio", SHAPES)
@pytest.mark.parametrize("cold", [0, 4])
def test_append_stores_the_documented_bytes(hga, dtype, d, kv, ratio, cold):
    sc = Scene(hga, dtype, d, kv, ratio, lens=(131, 1, 64, 200), cold=cold, layers=3, layer=1, seed=d + kv)
    # sequences' tokens from any position on, idle tokens between, one absent page
    runs = [(3, 150, 200), (-1, 4, 6), (0, 60, 131), (2, 63, 64), (9, 0, 1), (1, 0, 1), (0, 10 ** 6, 10 ** 6 + 2)]
    seq = np.concatenate([[s] * (b - a) for s, a, b in runs])
    pos = np.concatenate([np.arange(a, b) for _, a, b in runs])
    pos[50] = -5
    sc.table[3, 2] = sc.n_ids + 3  # positions 128..191 of sequence 3 have no page
    batch = sc.batch(seq, pos)
    T = len(seq)
    x = torch.from_numpy(_special(sc.rng, T, 2 * kv, d)).to(U.DT[dtype]).cuda()
    k, v = x[:, :kv], x[:, kv:]     # parts of one projection's rows
    want, kn, vn = sc.bytes.copy(), f64(k), f64(v)
    read = np.zeros((2, T, kv, d))
    closed = []
    for t in range(T):
        s, p = seq[t], pos[t]
        if not (0 <= s < 4 and 0 <= p < sc.max_pages * PAGE):
            continue
        pid = sc.table[s, p // PAGE]
        if not 0 <= pid < sc.n_ids:
            continue
        for h in range(kv):
            U.write_row(want[pid, h], d, p % PAGE, kn[t, h], vn[t, h])
        for i, y in enumerate((kn, vn)):
            read[i, t] = U.values(*U.quantise(y[t]))
        if p % PAGE == PAGE - 1:
            closed.append(pid)
    assert len(closed) == 3
    hga.hga_cache_append(sc.plan, sc.pool, 1, batch, k, v)
    assert np.array_equal(sc.stored(), want)
    assert (sc.pool.pages[0] == 255).all() and (sc.pool.pages[2] == 255).all()
    # summaries of the filled pages alone
    got = f64(sc.pool.page_sum[1])
    others = [i for i in range(sc.n_ids) if i not in closed]
    assert np.array_equal(got[others], sc.sums[others].astype(np.float64))
    n_hf = sc.plan.params.hf_pairs_chunk
    for pid in closed:
        kk = U.page_values(want[pid], d)[0]
        ref = U.summary(kk, d, sc.base, n_hf)
        # 64 additions of terms of two products with two rounded phases each
        mag = np.abs(kk).sum(-2) / PAGE
        mag = np.tile(mag[:, :d // 2] + mag[:, d // 2:], (1, 2))
        bad = np.isnan(ref)
        assert np.array_equal(np.isnan(got[pid]), bad)
        with np.errstate(invalid="ignore"):
            assert ((np.abs(got[pid] - ref) <= 80 * 2.0 ** -24 * mag) | bad).all()
    out = [torch.full((T, kv, d), 7.0, dtype=U.DT[dtype], device="cuda") for _ in range(2)]
    hga.hga_cache_read(sc.plan, sc.pool, 1, batch, *out)
    for o, r in zip(out, read):
        assert np.array_equal(f64(o), r, equal_nan=True)


@pytest.mark.parametrize("dtype,d,kv", [("bf16", 128, 2), ("f32", 64, 3)])
def test_tokens_one_by_one_are_the_prompt(hga, dtype, d, kv):
    n = 150
    one, all_ = (Scene(hga, dtype, d, kv, 2, lens=(n,), seed=3) for _ in range(2))
    k, v = one.random(n, kv, d), one.random(n, kv, d)
    hga.hga_cache_append(all_.plan, all_.pool, 0, all_.batch([0] * n, range(n)), k, v)
    for a in range(n):
        hga.hga_cache_append(one.plan, one.pool, 0, one.batch([0], [a]), k[a:a + 1], v[a:a + 1])
    assert np.array_equal(one.stored(), all_.stored())
    assert torch.equal(one.pool.page_sum, all_.pool.page_sum)
    # ... in any order
    o = torch.from_numpy(one.rng.permutation(n))
    mixed = Scene(hga, dtype, d, kv, 2, lens=(n,), seed=3)
    hga.hga_cache_append(mixed.plan, mixed.pool, 0, mixed.batch([0] * n, o.numpy()), k[o.cuda()], v[o.cuda()])
    assert np.array_equal(mixed.stored(), all_.stored())
    assert torch.equal(mixed.pool.page_sum, all_.pool.page_sum)
    # a rejected draft: positions appended again hold what was appended last
    k2, v2 = one.random(100, kv, d), one.random(100, kv, d)
    for a, b in ((50, 75), (75, 100), (100, 102), (102, 150)):
        hga.hga_cache_append(one.plan, one.pool, 0, one.batch([0] * (b - a), range(a, b)), k2[a - 50:b - 50],
                             v2[a - 50:b - 50])
    hga.hga_cache_append(all_.plan, all_.pool, 0, all_.batch([0] * 150, range(n)), torch.cat((k[:50], k2)),
                         torch.cat((v[:50], v2)))
    assert np.array_equal(one.stored(), all_.stored())
    assert torch.equal(one.pool.page_sum, all_.pool.page_sum)


@pytest.mark.parametrize("dtype,d,kv,layers,cold", [("bf16", 128, 4, 3, 5), ("f32", 64, 1, 1, 0), ("bf16", 64, 3, 2, 2)])
def test_copied_pages(hga, dtype, d, kv, layers, cold):
    sc = Scene(hga, dtype, d, kv, 1, lens=(600,), spare=9, cold=cold, layers=layers)
    n = sc.n_ids
    pool = sc.pool
    pool.pages.random_(0, 256)
    pool.page_sum.normal_()
    if cold:
        pool.cold.random_(0, 256)
    order = sc.rng.permutation(n)
    src, dst = order[:n // 2].astype(np.int32), order[n // 2:2 * (n // 2)].astype(np.int32)
    dst[1], src[2], src[3] = n, -1, 2 ** 31 - 1   # no pages: nothing happens
    dst[4] = src[4]
    both = torch.cat([pool.pages.cpu()] + ([pool.cold.clone()] if cold else []), 1)
    sums = pool.page_sum.clone().cpu()
    for s, t in zip(src, dst):
        if 0 <= s < n and 0 <= t < n:
            both[:, t], sums[:, t] = both[:, s].clone(), sums[:, s].clone()
    hga.hga_copy_pages(sc.plan, pool, torch.tensor(src).cuda(), torch.tensor(dst).cuda())
    torch.cuda.synchronize()
    now = torch.cat([pool.pages.cpu()] + ([pool.cold] if cold else []), 1)
    assert torch.equal(now, both) and torch.equal(pool.page_sum.cpu(), sums)


# ----------------------------------------------------------------- routing ---

def _route_check(sc, batch, q, extra=0):
    got = sc.route(batch, q, extra).cpu().numpy()
    want = U.route(f64(q), f64(sc.pool.page_sum[sc.layer]), sc.table, sc.seq, sc.pos, sc.kv, sc.first, sc.window,
                   sc.topk, got.shape[2], sc.n_ids)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("dtype,d,kv,ratio", SHAPES)
@pytest.mark.parametrize("first,last,prev,topk", [(1, 0, 1, 3), (2, 3, 1, 20), (0, 0, 0, 1), (0, 2, 0, 512)])
def test_listed_chunks(hga, dtype, d, kv, ratio, first, last, prev, topk):
    lens = (1, 64, 65, 700, 5000, 129, 2100)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, first=first, last=last, prev=prev, topk=topk, cold=7, layers=2,
               layer=1)
    seq = [s for s, n in enumerate(lens) for _ in range(3)] + [-1, 7, 4, 4]
    pos = [p for n in lens for p in (n - 1, (n - 1) // 2, 0)] + [0, 0, -1, 2 ** 31 - 1]
    batch = sc.batch(seq, pos)
    _route_check(sc, batch, sc.random(len(seq), sc.hq, d))
    # padded heads behind the queries: strided rows; a wider list
    wide = sc.random(len(seq), sc.hq + 2, d)
    _route_check(sc, batch, wide[:, :sc.hq], extra=5)
    # few tokens of long histories
    batch = sc.batch([4], [4999])
    _route_check(sc, batch, wide[:1, :sc.hq])


def test_a_prompts_tokens_route_alone(hga):
    sc = Scene(hga, "bf16", 64, 2, 4, lens=(1500, 300), topk=4)
    seq, pos = [0] * 1500 + [1] * 300, list(range(1500)) + list(range(300))
    _route_check(sc, sc.batch(seq, pos), sc.random(1800, sc.hq, 64))
    # of a longer history: more chunks than a wavefront has lanes
    sc = Scene(hga, "f32", 64, 2, 1, lens=(12001,), topk=40, last=2)
    _route_check(sc, sc.batch([0] * 1100, range(12001 - 1100, 12001)), sc.random(1100, sc.hq, 64))


def test_equal_scores_go_to_the_lowest_chunk(hga):
    sc = Scene(hga, "bf16", 64, 2, 2, lens=(64 * 40, 64 * 700), topk=5)
    sc.pool.page_sum.copy_(sc.pool.page_sum[:, :1].expand_as(sc.pool.page_sum).clone())
    q = sc.random(2, sc.hq, 64)
    _route_check(sc, sc.batch([0, 1], [64 * 40 - 1, 64 * 700 - 1]), q)
    _route_check(sc, sc.batch([0, 1], [64 * 40 - 1, 64 * 700 - 1]), torch.zeros_like(q))
    # a page that stands twice in a sequence, and one a hair above
    sc.pool.page_sum.normal_()
    sc.table[0, 3:30] = sc.table[0, 3]
    sc.table[1, ::2] = sc.table[1, 10]
    _route_check(sc, sc.batch([0, 1], [64 * 40 - 1, 64 * 700 - 1]), q)


def test_scores_an_fp32_sum_cannot_tell_apart(hga):
    """Summaries one fp32 step apart in one dimension, far from it in sum: the
    order of the 64-bit sums decides."""
    sc = Scene(hga, "f32", 128, 1, 2, lens=(64 * 300,), topk=17)
    ids = sc.table[0]
    base = np.float32(1000.0)
    step = np.arange(300, dtype=np.float32)
    x = np.full((300, 128), base, np.float32)
    x[:, 5] = 1.0 + sc.rng.permutation(step) * 2.0 ** -23
    sc.pool.page_sum[0, torch.tensor(ids).long(), 0] = torch.from_numpy(x).cuda()
    _route_check(sc, sc.batch([0], [64 * 300 - 1]), torch.ones(1, 2, 128, device="cuda"))


@pytest.mark.parametrize("pages,copies", [(60, 1), (60, 400), (130, 400), (700, 1), (700, 60), (1100, 1)])
def test_absent_pages_and_odd_summaries(hga, pages, copies):
    """In every form: few tokens and many, short histories and long."""
    sc = Scene(hga, "bf16", 128, 2, 3, lens=(64 * pages, 64 * 20), topk=6, last=2)
    sc.table[0, 5:20] = -1
    sc.table[0, [0, pages - 3, pages - 1]] = [sc.n_ids, 2 ** 31 - 1, -2 ** 31]
    sc.table[1, 1:17] = -1
    sums = sc.pool.page_sum[0]
    for i, x in zip((25, 30, 33, 41), (float("nan"), float("inf"), -float("inf"), 3e38)):
        sums[int(sc.table[0, i])] = x
    q = sc.random(3 * copies, sc.hq, 128)
    q[2] = q[2].abs() + 0.1
    q[1::5] = 0   # scores all equal, but for those that are not numbers
    _route_check(sc, sc.batch([0, 1, 0] * copies, [64 * pages - 1, 64 * 20 - 1, 64 * pages - 1] * copies), q)


@pytest.mark.parametrize("tokens,pages", [(1, 16400), (2, 16400), (40, 16400), (1, 70001)])
def test_histories_of_a_million_tokens(hga, tokens, pages):
    """16,400 and more chunks (over pages that recur): the workspace form."""
    n = pages + tokens
    sc = Scene(hga, "bf16", 64, 2, 2, lens=(64 * 500,), topk=9, max_pages=n)
    sc.table[0] = sc.table[0, sc.rng.integers(0, 500, n)]
    sc.sums = None
    pos = [64 * n - 1 - 64 * i for i in range(tokens)][::-1]
    _route_check(sc, sc.batch([0] * tokens, pos), sc.random(tokens, sc.hq, 64))


# --------------------------------------------------------------- attention ---

@pytest.mark.parametrize("dtype,d,kv,ratio", SHAPES)
def test_attention_over_whole_histories(hga, dtype, d, kv, ratio):
    lens = (1, 63, 64, 65, 130, 777, 2, 1600)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, layers=2, layer=1, seed=1)
    seq = list(range(8)) + [-1, 8, 5, 5, 7]
    pos = [n - 1 for n in lens] + [3, 0, -1, 10 ** 7, 800]
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, d, scale=1.5)
    got = sc.attend(batch, q)
    sc.check_attend(q, got)
    assert _same(got, sc.attend(batch, q))
    sc.check_attend(q, sc.attend(batch, q, workspace=False))
    wide = torch.zeros(len(seq), sc.hq + 3, d, dtype=q.dtype, device="cuda")
    wide[:, :sc.hq] = q
    assert _same(got, sc.attend(batch, wide[:, :sc.hq]))


@pytest.mark.parametrize("dtype,d,kv,ratio", SHAPES)
def test_attention_over_listed_pages(hga, dtype, d, kv, ratio):
    lens = (1, 64, 700, 1500, 129)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, cold=5, seed=2)
    sc.table[3, 4:9] = [-1, sc.n_ids, 2 ** 31 - 1, -2 ** 31, sc.table[3, 3]]
    seq = [0, 1, 2, 3, 4, 3, 3, 2, -1]
    pos = [0, 63, 699, 1499, 128, 700, 64, 640, 5]
    batch = sc.batch(seq, pos)
    T, n = len(seq), 9
    # chunks of the past and the future, repeated, missing, in any order; a row of none
    lists = sc.rng.integers(-3, 26, (T, kv, n)).astype(np.int32)
    lists[6] = -1
    lists[3, 0] = [2 ** 31 - 1, -2 ** 31, 23, 23, 5, 8, 3, 0, 99]
    lt = torch.from_numpy(lists).cuda()
    q = sc.random(T, sc.hq, d, scale=1.5)
    got = sc.attend(batch, q, lt)
    sc.check_attend(q, got, lt)
    assert _same(got, sc.attend(batch, q, lt))
    # the lists of the routing itself
    own = sc.route(batch, q)
    sc.check_attend(q, sc.attend(batch, q, own), own)


@pytest.mark.parametrize("dtype,d,kv,ratio,new", [
    ("bf16", 128, 2, 8, 100), ("bf16", 64, 1, 3, 70), ("f32", 64, 2, 1, 65), ("f32", 128, 1, 16, 5),
    ("bf16", 128, 1, 1, 129), ("bf16", 64, 2, 16, 33), ("bf16", 128, 1, 5, 17)])
def test_tokens_of_one_sequence_see_their_own_past(hga, dtype, d, kv, ratio, new):
    """Prompts, drafts and single tokens in one call, each token up to itself."""
    lens = (300, 64, 5, 900, 200)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=4)
    runs = [(3, lens[3] - new, lens[3]), (2, 4, 5), (1, 0, 64), (-1, 0, 3), (0, 290, 300), (4, 100, 104), (4, 150, 160)]
    seq = np.concatenate([[s] * (b - a) for s, a, b in runs])
    pos = np.concatenate([np.arange(a, b) for _, a, b in runs])
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, d)
    sc.check_attend(q, sc.attend(batch, q))
    # in another order the tokens give the same, to the order of sums
    o = sc.rng.permutation(len(seq))
    qo = q[torch.from_numpy(o).cuda()].contiguous()
    batch = sc.batch(seq[o], pos[o])
    sc.check_attend(qo, sc.attend(batch, qo))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_after_a_long_history(hga, dtype):
    sc = Scene(hga, dtype, 128, 1, 4, lens=(64 * 300 + 5,), seed=5)
    batch = sc.batch([0], [64 * 300 + 4])
    q = sc.random(1, 4, 128, scale=2.0)
    full = sc.attend(batch, q)
    sc.check_attend(q, full)
    nb = hga.hga_attend_tokens_workspace(sc.plan, batch)
    for part in (16, nb // 3 // 16 * 16, nb + 4096):
        sc.check_attend(q, sc.attend(batch, q, workspace=max(part, 16)))


@pytest.mark.parametrize("dtype,d,kv,ratio,new", [("bf16", 128, 1, 4, 45), ("f32", 64, 2, 3, 40), ("f32", 128, 1, 6, 30),
                                                  ("bf16", 64, 2, 16, 7)])
def test_a_draft_after_a_long_history(hga, dtype, d, kv, ratio, new):
    """Tokens that share their pages, the history cut into runs, some of its
    pages absent, some cold; with every size of workspace."""
    n = 64 * 90 + 11
    sc = Scene(hga, dtype, d, kv, ratio, lens=(n, 100, 64 * 70), cold=20, seed=7)
    sc.table[0, 20:31] = -1
    sc.table[2, [0, 69]] = sc.n_ids
    runs = [(0, n - new, n), (1, 90, 100), (2, 64 * 70 - new, 64 * 70)]
    seq = np.concatenate([[s] * (b - a) for s, a, b in runs])
    pos = np.concatenate([np.arange(a, b) for _, a, b in runs])
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, d)
    most = hga.hga_attend_tokens_workspace(sc.plan, batch)
    assert most > 0
    full = sc.attend(batch, q)
    sc.check_attend(q, full)
    assert _same(full, sc.attend(batch, q))
    for nb in (16, 4 * len(seq) + 16, most // 2 // 16 * 16, most + 64):
        sc.check_attend(q, sc.attend(batch, q, workspace=nb), tokens=slice(0, None, 7))


@pytest.mark.parametrize("dtype,ratio", [("bf16", 2), ("f32", 2), ("f32", 5)])
def test_thousands_of_units(hga, dtype, ratio):
    """More units than the device holds wavefronts: a wavefront each."""
    sc = Scene(hga, dtype, 64, 2, ratio, lens=(200, 65, 1, 400), seed=9)
    sc.table = np.tile(sc.table, (800, 1))
    lens = np.tile(sc.lens, 800)
    some = np.r_[0:40, 3000:3100, -30:0]
    # two tokens a sequence
    seq = np.repeat(np.arange(3200), 2)
    pos = np.stack((lens - 1, lens // 2), 1).reshape(-1)
    batch = sc.batch(seq, pos)
    q = sc.random(len(seq), sc.hq, 64)
    sc.check_attend(q, sc.attend(batch, q), tokens=some)
    sc.check_attend(q, sc.attend(batch, q, workspace=False), tokens=some)
    # lists of their own, in any order
    lists = torch.from_numpy(sc.rng.integers(-1, 8, (len(seq), 2, 5)).astype(np.int32)).cuda()
    sc.check_attend(q, sc.attend(batch, q, lists), lists, tokens=some)


def test_scores_far_apart_and_rows_that_are_not_numbers(hga):
    sc = Scene(hga, "bf16", 64, 2, 2, lens=(500, 500), seed=6)
    q = sc.random(2, 4, 64, scale=60.0)   # a weight of one, the rest far below
    batch = sc.batch([0, 1], [499, 499])
    sc.check_attend(q, sc.attend(batch, q))
    # a NaN key within sequence 0's past reaches every head over it, and nothing else
    pid = int(sc.table[0, 3])
    sc.pool.pages[0, pid, 0, U.addresses(64)[1][10, 0]] = 255
    out, lse = sc.attend(batch, q)
    assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all()
    assert not torch.isnan(out[0, 2:]).any() and not torch.isnan(out[1]).any()
    # and so does a NaN query
    q[1, 3, 9] = float("nan")
    out, lse = sc.attend(batch, q)
    assert torch.isnan(out[1, 3]).all() and not torch.isnan(out[1, :3]).any()


def test_pages_beyond_four_gigabytes(hga):
    """Offsets past 32 bits, in pages and in summaries."""
    d, kv = 128, 8
    plan = hga.Plan(batch=1, n_q_heads=kv, n_kv_heads=kv, head_dim=d, topk_chunks=2, topk_groups=4)
    n = (1 << 32) // (kv * U.head_bytes(d)) + 1100000 // 1024
    n = max(n, (1 << 32) // (kv * d * 4) // 8)
    pool = hga.Pool(plan, pages=torch.empty(1, n, kv, U.head_bytes(d), dtype=torch.uint8, device="cuda"),
                    page_sum=torch.empty(1, n, kv, d, device="cuda"))
    assert pool.pages.numel() > 1 << 32
    table = torch.tensor([[n - 1, n - 5], [2, 3]], dtype=torch.int32, device="cuda")
    seq = torch.tensor([s for s in (0, 1) for _ in range(100)], dtype=torch.int32, device="cuda")
    pos = torch.arange(100, dtype=torch.int32, device="cuda").repeat(2)
    batch = hga.TokenBatch(seq, pos, table)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn(100, kv, d, device="cuda", generator=g).bfloat16().repeat(2, 1, 1) for _ in range(3))
    hga.hga_cache_append(plan, pool, 0, batch, k, v)
    out = torch.empty_like(q)
    hga.hga_attend_tokens(plan, pool, 0, batch, q, out)
    assert torch.equal(out[:100], out[100:])
    assert torch.equal(pool.page_sum[0, n - 1], pool.page_sum[0, 2])
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    hga.hga_copy_pages(plan, pool, i32(n - 1, n - 5), i32(7, n - 2))
    table.copy_(torch.tensor([[7, n - 2], [2, 3]]))
    again = torch.empty_like(q)
    hga.hga_attend_tokens(plan, pool, 0, batch, q, again)
    assert torch.equal(out, again)
    rows = [torch.empty_like(k) for _ in range(2)]
    hga.hga_cache_read(plan, pool, 0, batch, *rows)
    assert torch.equal(rows[0][:100], rows[0][100:]) and torch.equal(rows[1][:100], rows[1][100:])


# ------------------------------------------------- streams, graphs, refusals ---

def test_other_streams_and_replayed_graphs(hga):
    """A decode step captured once and replayed for step after step, tokens and
    positions changed in place, against the same steps run eagerly."""
    lens = (200, 64, 1000, 7)
    a, b = (Scene(hga, "bf16", 128, 2, 4, lens=[n + 70 for n in lens], topk=3, seed=8) for _ in range(2))
    steps = 70
    g = torch.Generator().manual_seed(5)
    qs, ks, vs = (torch.randn(steps, 4, h, 128, generator=g).bfloat16().cuda() for h in (8, 2, 2))

    def make(sc):
        batch = sc.batch([0, 1, 2, 3], lens)
        st = dict(batch=batch, q=qs[0].clone(), k=ks[0].clone(), v=vs[0].clone(), out=torch.zeros_like(qs[0]),
                  lse=torch.zeros(4, 8, device="cuda"),
                  lists=torch.zeros(4, 2, hga.hga_token_list_size(sc.plan), dtype=torch.int32, device="cuda"))
        st["ws"] = torch.empty(max(16, hga.hga_attend_tokens_workspace(sc.plan, batch, st["lists"])),
                               dtype=torch.uint8, device="cuda")
        return st

    def step(sc, st):
        hga.hga_cache_append(sc.plan, sc.pool, 0, st["batch"], st["k"], st["v"])
        hga.hga_route_tokens(sc.plan, sc.pool, 0, st["batch"], st["q"], st["lists"])
        hga.hga_attend_tokens(sc.plan, sc.pool, 0, st["batch"], st["q"], st["out"], lse=st["lse"],
                              chunk_list=st["lists"], workspace=st["ws"])

    sa, sb = make(a), make(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(b, sb)
    for i in range(steps):
        for st in (sa, sb):
            for n, x in (("q", qs), ("k", ks), ("v", vs)):
                st[n].copy_(x[i])
        if i % 2:
            with torch.cuda.stream(side):
                side.wait_stream(torch.cuda.default_stream())
                step(a, sa)
            torch.cuda.default_stream().wait_stream(side)
        else:
            step(a, sa)
        graph.replay()
        assert torch.equal(sa["lists"], sb["lists"])
        assert _same((sa["out"], sa["lse"]), (sb["out"], sb["lse"]))
        for st in (sa, sb):
            st["batch"].tok_pos.add_(1)
    assert np.array_equal(a.stored(), b.stored())
    assert torch.equal(a.pool.page_sum, b.pool.page_sum)


def test_replays_find_nothing_in_their_workspace(hga):
    """A captured call over a split history, tokens sharing pages: replayed with
    other positions and queries, its workspace filled with anything between."""
    n = 64 * 80
    sc = Scene(hga, "bf16", 128, 1, 4, lens=(n, n), seed=10)
    seq = torch.tensor([0] * 9 + [1] * 5, dtype=torch.int32)
    pos = torch.arange(14, dtype=torch.int32) + n - 40
    batch = sc.batch(seq.numpy(), pos.numpy())
    q, out = sc.random(14, 4, 128), torch.zeros(14, 4, 128, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(14, 4, device="cuda")
    lists = torch.zeros(14, 1, hga.hga_token_list_size(sc.plan), dtype=torch.int32, device="cuda")
    nb = hga.hga_attend_tokens_workspace(sc.plan, batch)
    ws = torch.zeros(nb, dtype=torch.uint8, device="cuda")
    rws = torch.zeros(max(hga.hga_route_tokens_workspace(sc.plan, batch), 16), dtype=torch.uint8, device="cuda")

    def calls(out, lse, lists):
        hga.hga_route_tokens(sc.plan, sc.pool, 0, batch, q, lists, workspace=rws)
        hga.hga_attend_tokens(sc.plan, sc.pool, 0, batch, q, out, lse=lse, workspace=ws)

    calls(out, lse, lists)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(out, lse, lists)
    for i in range(5):
        q.copy_(sc.random(14, 4, 128))
        batch.tok_pos.add_(3)
        batch.tok_seq.copy_(seq.roll(i))
        ws.fill_(255 - i)
        rws.random_()
        graph.replay()
        eager = torch.empty_like(out), torch.empty_like(lse), torch.empty_like(lists)
        calls(*eager)
        assert _same((out, lse), eager[:2]) and torch.equal(lists, eager[2])
        sc.seq, sc.pos = batch.tok_seq.cpu().numpy(), batch.tok_pos.cpu().numpy()
        sc.check_attend(q, (out, lse))


def test_no_tokens_and_empty_tables(hga):
    sc = Scene(hga, lens=(70,))
    for seq, pos in (([], []), ([0, 0], [1, 2])):
        for shape in ((0, 3), (2, 0), (0, 0)):
            b = hga.TokenBatch(torch.tensor(seq, dtype=torch.int32).cuda(), torch.tensor(pos, dtype=torch.int32).cuda(),
                               torch.zeros(shape, dtype=torch.int32, device="cuda"))
            q = torch.ones(len(seq), sc.hq, sc.d, dtype=torch.bfloat16, device="cuda")
            before = sc.stored()
            hga.hga_cache_append(sc.plan, sc.pool, 0, b, q[:, :2], q[:, :2])
            assert np.array_equal(before, sc.stored())
            assert (sc.route(b, q) == -1).all()
            out, lse = sc.attend(b, q)
            assert (out == 0).all() and (lse == -np.inf).all()
    hga.hga_copy_pages(sc.plan, sc.pool, b.tok_seq[:0], b.tok_seq[:0])
    # a pool without a page
    none = hga.Pool(sc.plan, 0)
    b = sc.batch([0, 0], [69, 5])
    sc.pool = none
    hga.hga_cache_append(sc.plan, none, 0, b, q[:, :2], q[:, :2])
    assert (sc.route(b, q) == -1).all()
    out, lse = sc.attend(b, q)
    assert (out == 0).all() and (lse == -np.inf).all()
    hga.hga_copy_pages(sc.plan, none, b.tok_seq, b.tok_pos)


def test_refusals(hga):
    sc = Scene(hga, lens=(70, 70), cold=1)
    b = sc.batch([0, 1], [69, 69])
    q, k = sc.random(2, sc.hq, 64), sc.random(2, sc.kv, 64)
    n = hga.hga_token_list_size(sc.plan)
    lists = torch.zeros(2, sc.kv, n, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    odd = torch.empty(2 * sc.hq * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:]
    off = odd[:2 * sc.hq * 64].view(2, sc.hq, 64)           # not 16-byte aligned
    step = torch.empty(2, sc.hq * 64 + 1, dtype=torch.bfloat16, device="cuda")[:, :sc.hq * 64].view(2, sc.hq, 64)
    append = lambda **x: hga.hga_cache_append(sc.plan, x.get("pool", sc.pool), x.get("layer", 0),  # noqa: E731
                                              x.get("b", b), x.get("k", k), x.get("v", k))
    route = lambda **x: hga.hga_route_tokens(sc.plan, sc.pool, x.get("layer", 0), b, x.get("q", q),  # noqa: E731
                                             x.get("lists", lists))
    att = lambda **x: hga.hga_attend_tokens(sc.plan, sc.pool, x.get("layer", 0), b, x.get("q", q),  # noqa: E731
                                            x.get("out", out), lse=x.get("lse"), chunk_list=x.get("lists"),
                                            workspace=x.get("ws"))
    copy = lambda s, t: hga.hga_copy_pages(sc.plan, sc.pool, s, t)  # noqa: E731
    read = lambda **x: hga.hga_cache_read(sc.plan, sc.pool, x.get("layer", 0), b, x.get("k", k), k)  # noqa: E731
    i32 = torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = [
        (append, dict(layer=1)), (append, dict(layer=-1)), (append, dict(k=k.float())), (append, dict(k=k[:1])),
        (append, dict(v=k.cpu())), (append, dict(k=k.transpose(0, 1))), (append, dict(v=q[:, ::2])),
        (read, dict(k=q)), (read, dict(layer=2)), (route, dict(lists=lists[..., :n - 1].contiguous())),
        (route, dict(lists=lists.long())), (route, dict(lists=lists[..., ::2])), (route, dict(q=off)),
        (route, dict(q=step)), (route, dict(q=k)), (att, dict(q=off)), (att, dict(out=off)),
        (att, dict(out=out.float())), (att, dict(lse=torch.empty(2, sc.hq + 1, device="cuda"))),
        (att, dict(lists=lists[..., :0])), (att, dict(lists=lists[:1])), (att, dict(ws=odd)),
        (att, dict(lists=lists.cpu())), (att, dict(layer=1)),
    ]
    sc.pool.pages.fill_(3)
    for f, kw in bad:
        with pytest.raises(hga.HgaError) as e:
            f(**kw)
        assert e.value.status in (-1, -2, -3), kw
    for s, t in ((i32, i32[:2]), (i32.long(), i32), (i32.cpu(), i32.cpu())):
        with pytest.raises(hga.HgaError):
            copy(s, t)
    other = hga.Plan(batch=1, n_q_heads=2, n_kv_heads=2, head_dim=128, topk_chunks=1, topk_groups=1)
    for make in (lambda: hga.hga_copy_pages(other, sc.pool, i32, i32),
                 lambda: hga.hga_cache_append(other, sc.pool, 0, b, q[..., :1], q[..., :1]),
                 lambda: hga.Pool(sc.plan, pages=sc.pool.pages[..., :-1].contiguous()),
                 lambda: hga.Pool(sc.plan, pages=sc.pool.pages.cpu()),
                 lambda: hga.Pool(sc.plan, pages=sc.pool.pages, cold=sc.pool.cold.clone()),
                 lambda: hga.Pool(sc.plan, pages=sc.pool.pages, page_sum=sc.pool.page_sum[:, :1].contiguous()),
                 lambda: hga.TokenBatch(b.tok_seq, b.tok_pos[:1], b.page_table),
                 lambda: hga.TokenBatch(b.tok_seq.long(), b.tok_pos, b.page_table),
                 lambda: hga.TokenBatch(b.tok_seq, b.tok_pos, b.page_table.t()),
                 lambda: hga.TokenBatch(b.tok_seq.cpu(), b.tok_pos.cpu(), b.page_table.cpu())):
        with pytest.raises(hga.HgaError):
            make()
    torch.cuda.synchronize()
    assert (sc.pool.pages == 3).all()


# ---------------------------------------------------- the operators together ---

class _Twin:
    """A PagedCache served token by token beside plain copies of what was
    appended (as stored), attended in 64 bits."""

    def __init__(self, hga, dtype, d, kv, ratio, routed, layers=2, topk=3, n_cold=6):
        from paper_2606_30709_amd.pages import PagedCache
        from paper_2606_30709_amd.pipeline import TokenPipeline
        self.hga, self.dtype, self.d, self.kv, self.hq, self.routed = hga, dtype, d, kv, kv * ratio, routed
        self.plan = hga.Plan(batch=1, n_q_heads=self.hq, n_kv_heads=kv, head_dim=d, keep_first=1, keep_last=1,
                             topk_chunks=topk, topk_groups=4, dtype=hga.F32 if dtype == "f32" else hga.BF16)
        self.cache = PagedCache(self.plan, 90, 4, 20, n_layers=layers, n_cold=n_cold)
        self.pipe = TokenPipeline(self.cache, routed)
        self.layers = layers
        self.kept = [[[np.zeros((2, 0, kv, d))] for _ in range(layers)] for _ in range(4)]
        self.rng = np.random.default_rng(3)
        self.topk = topk

    def rand(self, *s):
        return torch.from_numpy(self.rng.standard_normal(s).astype(np.float32)).to(U.DT[self.dtype]).cuda()

    def serve(self, seqs, counts, check=True):
        batch = self.cache.append(seqs, counts)
        T, hga = batch.n_tokens, self.hga
        seq, pos = (x.cpu().numpy().astype(np.int64) for x in (batch.tok_seq, batch.tok_pos))
        table = self.cache.page_table.cpu().numpy()
        assert np.array_equal(table, self.cache.book.table)
        results = []
        for layer in range(self.layers):
            q, k, v = self.rand(T, self.hq, self.d), self.rand(T, self.kv, self.d), self.rand(T, self.kv, self.d)
            out, lse = self.pipe.step(layer, batch, q, k, v)
            results.append((out.clone(), lse.clone()))
            rows = [U.values(*U.quantise(f64(x))) for x in (k, v)]
            for s in set(seq.tolist()):
                self.kept[s][layer][0] = np.concatenate((self.kept[s][layer][0], np.stack([r[seq == s] for r in rows])), 1)
            if not check:
                continue
            # pages rebuilt from what was appended
            ids = self.cache.pool.n_pages + self.cache.pool.n_cold
            kp, vp = np.zeros((2, ids, self.kv, PAGE, self.d))
            for s in range(4):
                x = self.kept[s][layer][0]
                for c in range(-(-x.shape[1] // PAGE)):
                    part = x[:, c * PAGE:(c + 1) * PAGE].transpose(0, 2, 1, 3)
                    if table[s, c] >= 0:
                        kp[table[s, c], :, :part.shape[2]], vp[table[s, c], :, :part.shape[2]] = part
            lists = None
            if self.routed:
                sums = U.summary(kp, self.d, 10000.0, self.plan.params.hf_pairs_chunk)
                n_list = hga.hga_token_list_size(self.plan)
                lists = U.route(f64(q), sums, table, seq, pos, self.kv, 1, 1, self.topk, n_list, ids)
                got = self.pipe._buffer("lists", (T, self.kv, n_list), torch.int32).cpu().numpy()
                assert np.array_equal(got, lists)
            ref, rlse, mag, reach, count = U.attend(f64(q), kp, vp, table, seq, pos, self.kv, lists, ids)
            tol, ltol = U.attend_tolerance(self.dtype, self.d, ref, mag, reach, count)
            assert (np.abs(f64(out) - ref) <= tol).all() and (np.abs(f64(lse) - rlse) <= ltol).all()
        return results


@pytest.mark.parametrize("dtype,d,kv,ratio,routed", [("bf16", 128, 2, 4, True), ("f32", 64, 2, 1, True),
                                                     ("bf16", 64, 3, 2, False)])
def test_serving_a_batch_of_sequences(hga, dtype, d, kv, ratio, routed):
    """Prompts, single tokens, forks, drafts taken back, pages dropped, moved to
    the cold tier and back, and moved together."""
    t = _Twin(hga, dtype, d, kv, ratio, routed)
    cache = t.cache
    t.serve([], [])
    t.serve([1], [0])
    t.serve([2, 0], [300, 450])
    t.serve([0, 2], [1, 1])
    cache.fork(0, 1)
    t.kept[1] = [[x[0].copy()] for x in t.kept[0]]
    t.serve([1, 0, 2], [1, 1, 70])
    cache.truncate(0, 400)
    t.kept[0] = [[x[0][:, :400]] for x in t.kept[0]]
    t.serve([0, 1], [3, 2])
    assert cache.to_cold(1, 1, 6) == 5
    t.serve([2, 1, 0], [1, 1, 200])
    cache.drop(2, 1, 3)
    cache.release(0)
    t.kept[0] = [[x[0][:, :0]] for x in t.kept[0]]
    t.serve([1, 2], [60, 1])
    assert cache.compact() > 0
    t.serve([2, 3, 1], [1, 130, 1])
    assert cache.to_device(1, 0, 6) == 5
    t.serve([1, 2, 3], [1, 1, 1])


def test_moved_pages_give_the_same_bits(hga):
    """Where pages lie changes nothing: compaction, the cold tier, a fork."""
    t = _Twin(hga, "bf16", 128, 2, 4, True, n_cold=12)
    cache = t.cache
    t.serve([0, 1, 3], [333, 100, 700], check=False)
    cache.release(1)
    cache.fork(0, 2)

    def look(s):
        n = cache.length(s)
        one = lambda x: torch.tensor([x], dtype=torch.int32).cuda()  # noqa: E731
        batch = hga.TokenBatch(one(s), one(n - 1), cache.page_table)
        g = torch.Generator().manual_seed(1)
        q = torch.randn(1, t.hq, t.d, generator=g).bfloat16().cuda()
        out = []
        for layer in range(t.layers):
            lists = torch.zeros(1, t.kv, hga.hga_token_list_size(t.plan), dtype=torch.int32, device="cuda")
            hga.hga_route_tokens(t.plan, cache.pool, layer, batch, q, lists)
            for ls in (lists, None):
                o, l = torch.empty_like(q), torch.empty(1, t.hq, device="cuda")
                hga.hga_attend_tokens(t.plan, cache.pool, layer, batch, q, o, lse=l, chunk_list=ls)
                out += [o, l]
        return out

    first = look(0), look(3)
    assert _same(first[0], look(2))
    for change in (lambda: cache.to_cold(3, 0, 10), lambda: cache.compact(), lambda: cache.to_cold(0, 2, 4),
                   lambda: cache.to_device(3, 1, 9), lambda: cache.compact()):
        change()
        assert _same(first[0], look(0)) and _same(first[1], look(3)) and _same(first[0], look(2))
