"""Single tokens over the paged 4-bit cache where it can go wrong: the precision
of the weights, rows that are not numbers, keys that pile up at the border of a
selection, captured steps beside larger ones, wide tables."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import tokens_util as U
from test_tokens import _route_check
from tokens_util import Scene, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


# -------------------------------------------------------------- the weights ---

def _rounded_once(sc, q, got, lists=None):
    """A bf16 result carries one rounding of its own (2^-8 of it at most).  What
    comes before is in proportion to sum p |v| / l: a score's error as in
    tokens_util.attend_tolerance, the sums', and the weight's.  That one enters
    the product as two bf16 terms: the first leaves at most 2^-8 of it, the second
    2^-8 of that."""
    k, v = sc.k_v()
    ln = None if lists is None else lists.cpu().numpy()
    ref, _, mag, reach, count = U.attend(f64(q), k, v, sc.table, sc.seq, sc.pos, sc.kv, ln, sc.n_ids)
    u = 2.0 ** -24
    rel = 2 * (2 * (sc.d + 12) * u * reach + 8 * u) + 2 * count * u + 2.0 ** -16
    before = rel[..., None] * mag
    err = np.abs(f64(got[0]) - ref)
    tol = before + 2.0 ** -8 * (np.abs(ref) + before) + 1e-30
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("d,kv,ratio", [(128, 4, 8), (64, 3, 3), (64, 1, 16), (128, 5, 2), (128, 1, 1)])
def test_bf16_results_are_rounded_once(hga, d, kv, ratio):
    """Weights of about the same size over values of either sign: results far
    below the values, which a weight of eight bits would not carry.  In the
    forms of one token a unit, of several (one tile and two), of lists."""
    lens = (64, 130, 300, 7, 1)
    sc = Scene(hga, "bf16", d, kv, ratio, lens=lens, seed=11)
    single = sc.batch(range(5), [n - 1 for n in lens])
    q = sc.random(5, sc.hq, d, scale=0.05)
    _rounded_once(sc, q, sc.attend(single, q))
    lists = torch.from_numpy(np.tile(np.int32([0, 1, -1, 4]), (5, kv, 1))).cuda()
    _rounded_once(sc, q, sc.attend(single, q, lists), lists)
    for n in (3, 60):
        seq, pos = [0] * n + [1] * n + [2] * n, [*range(64 - n, 64), *range(130 - n, 130), *range(200, 200 + n)]
        q = sc.random(3 * n, sc.hq, d, scale=0.05)
        _rounded_once(sc, q, sc.attend(sc.batch(seq, pos), q))


@pytest.mark.parametrize("d,ratio", [(64, 1), (64, 5), (128, 4), (128, 16)])
def test_the_largest_fp32_queries(hga, d, ratio):
    """Queries up to the largest float over keys as small: scores of ordinary size."""
    sc = Scene(hga, "f32", d, 2, ratio, lens=(200, 70, 330), seed=15)
    ks = U.addresses(d)[1]
    sc.bytes[..., ks] = 2  # 2^-125
    sc.pool.pages[0].copy_(torch.from_numpy(sc.bytes))
    for seq, pos in (([0, 1, 2], [199, 69, 329]), ([0] * 9 + [2] * 40, [*range(191, 200), *range(290, 330)])):
        q = sc.random(len(seq), sc.hq, d)
        q = q * (2.0 ** 124 / d ** 0.5)
        q[:, :, 3], q[:, ::2, 17] = torch.finfo(torch.float32).max, -torch.finfo(torch.float32).max
        batch = sc.batch(seq, pos)
        sc.check_attend(q, sc.attend(batch, q))
        sc.check_attend(q, sc.attend(batch, q, workspace=False))


# --------------------------------------------------- rows that are not numbers ---

@pytest.mark.parametrize("dtype,d,kv,ratio,n", [
    ("bf16", 128, 2, 8, 3), ("bf16", 128, 2, 8, 70), ("bf16", 64, 1, 1, 100), ("bf16", 64, 2, 16, 5),
    ("bf16", 64, 1, 3, 200), ("f32", 128, 2, 2, 40), ("f32", 64, 2, 4, 70), ("f32", 64, 1, 16, 4)])
@pytest.mark.parametrize("pages", [3, 60])
def test_a_value_that_is_no_number_reaches_later_tokens_only(hga, dtype, d, kv, ratio, n, pages):
    """Value blocks that stand for NaN among the rows of a call's own tokens
    (tokens that share their pages, from one page to several behind, few pages and
    many): in the block's dimensions, tokens from that row on are NaN, and nothing
    else is, with a workspace (of any size) as without."""
    sc = Scene(hga, dtype, d, kv, ratio, lens=(64 * pages + 20, 40), seed=13)
    last = sc.lens[0]
    _, _, _, vs = U.addresses(d)
    clean = sc.k_v()
    # (position, head, block): the first and last of the call's tokens, one before them all, one twice in a row
    bad = [(last - n // 2, 0, 0), (last - 1, kv - 1, d // 32 - 1), (last - n + 1, 0, d // 32 - 1),
           (last - n // 3, kv - 1, 1), (last - n // 3, kv - 1, 0)]
    for p, h, b in bad:
        sc.pool.pages[0, int(sc.table[0, p // 64]), h, int(vs[p % 64, 32 * b])] = 255
    seq, pos = np.array([0] * n + [1] * 3), np.array([*range(last - n, last), 3, 39, 20])
    batch = sc.batch(seq, pos)
    q = sc.random(n + 3, sc.hq, d)
    want = np.zeros((n + 3, sc.hq, d), bool)
    for p, h, b in bad:
        want[:n][pos[:n] >= p, h * ratio:(h + 1) * ratio, 32 * b:32 * b + 32] = True
    ref, rlse, mag, reach, count = U.attend(f64(q), *clean, sc.table, seq, pos, kv, None, sc.n_ids)
    tol, ltol = U.attend_tolerance(dtype, d, ref, mag, reach, count)
    for ws in (True, 4 * (n + 3) + 32, False):
        out, lse = sc.attend(batch, q, workspace=ws)
        o, l = f64(out), f64(lse)
        assert np.array_equal(np.isnan(o), want)
        assert ((np.abs(o - ref) <= tol) | want).all()
        assert (np.abs(l - rlse) <= ltol).all()


# -------------------------------------------------------------- the routing ---

@pytest.mark.parametrize("tokens", [1, 70])
@pytest.mark.parametrize("low", ["close", "equal", "two"])
def test_more_keys_at_the_border_than_a_workgroup_ranks(hga, tokens, low):
    """More than 512 low scores under a few high ones, the border among them:
    apart from one another, equal, or of two values.  With one token the scores
    are formed by the whole device, with more by a workgroup a token and head."""
    pages = 1100
    sc = Scene(hga, "f32", 64, 2, 1, lens=(64 * pages,), topk=20, seed=12)
    x = {"close": 1.0 + sc.rng.permutation(pages) * 1e-6, "equal": np.ones(pages),
         "two": 1.0 + (np.arange(pages) % 2) * 1e-3}[low]
    x[[30, 500, 1000]] = [1000.0, 900.0, 1000.0]
    sums = np.zeros((pages, 2, 64), np.float32)
    sums[:, 0, 3], sums[:, 1, 60] = x, -x[::-1]
    sc.pool.page_sum[0, torch.from_numpy(sc.table[0]).long()] = torch.from_numpy(sums).cuda()
    q = torch.zeros(tokens, 2, 64, device="cuda")
    q[:, 0, 3], q[:, 1, 60] = 1.0, -1.0
    pos = [64 * pages - 1 - i for i in range(tokens)]
    _route_check(sc, sc.batch([0] * tokens, pos), q)


def test_many_tokens_through_a_wide_table(hga):
    """A table of 20,000 pages a sequence, for the sake of one: the keys' workspace
    stays small, and a call whose units it does not hold goes through it in parts."""
    from types import SimpleNamespace
    sc = Scene(hga, "bf16", 64, 3, 2, lens=(64 * 30, 64 * 500, 70), topk=6, max_pages=20000, seed=14)
    for n, pages in ((4096, 1 << 18), (1 << 20, 1 << 18), (700, 20000), (1 << 28, 16385)):
        assert 0 < hga.hga_route_tokens_workspace(sc.plan, SimpleNamespace(n_tokens=n, max_pages=pages)) <= 1 << 28
    sc.table[1] = sc.table[1, sc.rng.integers(0, 500, 20000)]  # over pages that recur
    n = 700                                                     # of which a part holds 559
    seq = np.array([0] * 690 + [1] * 2 + [2] * 8)
    pos = np.array([*range(64 * 30 - 690, 64 * 30), 64 * 19000 + 5, 64 * 20000 - 1, *range(62, 70)])
    order = sc.rng.permutation(n)
    batch = sc.batch(seq[order], pos[order])
    q = sc.random(n, sc.hq, 64)
    nb = hga.hga_route_tokens_workspace(sc.plan, batch)
    assert nb < 8 * 3 * n * 20000
    _route_check(sc, batch, q)
    # ... and in one part, to the same lists; a workspace below what is asked for is refused
    lists = [torch.full((n, 3, hga.hga_token_list_size(sc.plan)), -7, dtype=torch.int32, device="cuda") for _ in range(2)]
    for out, nbytes in zip(lists, (nb, 8 * 3 * n * 20000)):
        hga.hga_route_tokens(sc.plan, sc.pool, 0, batch, q, out,
                             workspace=torch.empty(nbytes, dtype=torch.uint8, device="cuda"))
    assert torch.equal(*lists)
    with pytest.raises(hga.HgaError):
        hga.hga_route_tokens(sc.plan, sc.pool, 0, batch, q, lists[0],
                             workspace=torch.empty(nb - 16, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------ captured steps ---

@pytest.mark.parametrize("routed", [True, False])
def test_a_captured_step_beside_larger_ones(hga, routed):
    """A decode step captured, a prompt run through the same pipeline, memory
    allocated and filled where its buffers might have been; then replays for the
    next tokens, against a pipeline of their own, and the filled memory as it
    was."""
    from paper_2606_30709_amd.pages import PagedCache
    from paper_2606_30709_amd.pipeline import TokenPipeline
    plan = hga.Plan(batch=1, n_q_heads=8, n_kv_heads=2, head_dim=128, keep_first=1, keep_last=1, topk_chunks=3,
                    topk_groups=4)
    cache = PagedCache(plan, 300, 4, 80, n_layers=2)
    pipe, other = TokenPipeline(cache, routed), TokenPipeline(cache, routed)
    g = torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g).bfloat16().cuda()  # noqa: E731

    def prompt(seqs, counts):
        b = cache.append(seqs, counts)
        for layer in (0, 1):
            pipe.step(layer, b, rand(b.n_tokens, 8, 128), rand(b.n_tokens, 2, 128), rand(b.n_tokens, 2, 128))

    prompt([0, 1, 2], [40, 4500, 30])
    pipe = TokenPipeline(cache, routed)  # of small steps so far
    batch = cache.append([0, 1, 2], [1, 1, 1])
    q, k, v = rand(3, 8, 128), rand(3, 2, 128), rand(3, 2, 128)
    step = lambda p: [p.step(layer, batch, q, k, v) for layer in (0, 1)][1]  # noqa: E731
    step(pipe)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(pipe)
    addresses = {t.data_ptr() for t in pipe._buf.values()}
    prompt([3], [700])
    assert not addresses & {t.data_ptr() for t in pipe._buf.values()}
    filled = [torch.full((n,), 77, dtype=torch.uint8, device="cuda") for n in [512] * 200 + [2 ** 20] * 40 + [2 ** 22] * 8]
    for _ in range(4):
        b = cache.append([0, 1, 2], [1, 1, 1])
        batch.tok_seq.copy_(b.tok_seq)
        batch.tok_pos.copy_(b.tok_pos)
        for x in (q, k, v):
            x.copy_(rand(*x.shape))
        graph.replay()
        want = step(other)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert all(bool((t == 77).all()) for t in filled)
    with pytest.raises(hga.HgaError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            step(TokenPipeline(cache, routed))
