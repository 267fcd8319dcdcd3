"""Values that are zero in hga_attend_shared: stored with the smallest scale, they
are no reason to leave the form for values that f16 holds."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import prefix_util as P
import tokens_util as U
from tokens_util import PAGE, Scene

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hga():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga as H
    H.library()
    return H


def _set(sc, d, page, rows, blocks, codes, scale):
    """Blocks of some rows' values: the codes' bytes and the scale."""
    _, _, vc, vs = U.addresses(d)
    for r in rows:
        for b in blocks:
            sc.bytes[page][:, vc[r, 32 * b:32 * b + 32]] = codes
            sc.bytes[page][:, vs[r, 32 * b]] = scale


@pytest.mark.parametrize("dtype,d,kv,ratio,n", [("bf16", 128, 2, 8, 30), ("bf16", 64, 1, 3, 60), ("bf16", 128, 1, 4, 9),
                                                ("f32", 64, 1, 1, 90)])
@pytest.mark.parametrize("few", [False, "few"])
def test_zeros_of_any_scale(hga, dtype, d, kv, ratio, n, few):
    """The same bits from zeros with the scale that appending gives them as from
    zeros with one in the middle of f16's range, and those of the definition: a
    block, a row, a page, everything; negative ones too."""
    pages, last = 19, d // 32 - 1
    lens = [PAGE * pages + 1 + i * 69 // (n - 1) for i in range(n)]
    assert U.quantise(np.zeros(d))[1].tolist() == [2] * (d // 32)
    for at in ([(4, [33], [last], 0)], [(2, [7], range(last + 1), 0x88), (9, range(PAGE), range(last + 1), 0), (18, [63], [0], 0x80)],
               [(c, range(PAGE), range(last + 1), 0) for c in range(pages)]):
        got = []
        for scale in (2, 127):
            sc = Scene(hga, dtype, d, kv, ratio, lens=lens, seed=n)
            P.share(sc, [(0, list(range(1, n)), pages)])
            for c, rows, blocks, codes in at:
                _set(sc, d, sc.table[0, c], rows, blocks, codes, scale)
            _set(sc, d, sc.table[3, pages], [0], [0], 0, scale)      # a token's own
            sc.pool.pages[0].copy_(torch.from_numpy(sc.bytes))
            seq = np.arange(n)
            batch = sc.batch(seq, [x - 1 for x in lens])
            q = sc.random(n, sc.hq, d)
            px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], sc.rng, own_hint=2)
            got.append(P.attend(sc, batch, px, q, share=few or True))
            P.check_attend(sc, q, got[-1], tokens=slice(0, 12))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("d,kv,ratio,n", [(128, 2, 8, 30), (64, 1, 3, 60)])
@pytest.mark.parametrize("few", [False, "few"])
def test_what_is_not_zero_beside_zeros(hga, d, kv, ratio, n, few):
    """One value that f16 does not hold (or that is no number) among zeros of such
    a scale, anywhere in its block."""
    pages = 9
    _, _, vc, vs = U.addresses(d)
    lens = [PAGE * pages + 1 + i for i in range(n)]
    for at, (scale, dim, code) in enumerate(((60, 0, 1), (60, 31, 0x10), (150, 17, 0x70), (2, 9, 0x90), (255, 0, 0))):
        sc = Scene(hga, "bf16", d, kv, ratio, lens=lens, seed=at)
        P.share(sc, [(0, list(range(1, n)), pages)])
        page, row, block = sc.table[0, 3], 21 + 9 * at, at % (d // 32)
        _set(sc, d, page, range(PAGE), range(d // 32), 0, 2)
        _set(sc, d, page, [row], [block], 0, scale)
        sc.bytes[page][:, vc[row, 32 * block + dim]] = code
        sc.pool.pages[0].copy_(torch.from_numpy(sc.bytes))
        seq = np.arange(n)
        batch = sc.batch(seq, [x - 1 for x in lens])
        q = sc.random(n, sc.hq, d)
        px = P.prefixes(hga, seq, {s: 0 for s in range(n)}, [pages], sc.rng, own_hint=2)
        out, lse = P.attend(sc, batch, px, q, share=few or True)
        if scale == 255:
            want = torch.zeros(d, dtype=torch.bool, device="cuda")
            want[32 * block:32 * block + 32] = True
            assert torch.equal(out.isnan(), want.expand_as(out)) and torch.isfinite(lse).all()
        else:
            P.check_attend(sc, q, (out, lse), tokens=slice(0, 12))
