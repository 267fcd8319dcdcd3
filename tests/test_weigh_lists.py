"""hga_weigh_pages over lists of more entries than a wavefront looks at once."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import prefix_util as P
from tokens_util import Scene

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,kv,ratio,n", [("bf16", 128, 2, 8, 64), ("f32", 64, 1, 3, 65), ("bf16", 64, 3, 1, 150), ("f32", 128, 1, 2, 193)])
def test_long_lists(dtype, d, kv, ratio, n):
    """Entries in any order, of no page, and of one page in several places; with
    slices of the tokens and without."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2606_30709_amd import hga
    lens = (64 * 100 + 3, 700, 64 * 40)
    sc = Scene(hga, dtype, d, kv, ratio, lens=lens, cold=7, seed=n)
    sc.table[0, 4:9] = [-1, sc.n_ids, 2 ** 31 - 1, -2 ** 31, sc.table[0, 3]]
    seq = np.array([0, 1, 2] * 5 + [0, -1])
    pos = np.array([max(lens[s] - 1 - 29 * i, 0) if s >= 0 else 3 for i, s in enumerate(seq)])
    batch = sc.batch(seq, pos)
    lists = sc.rng.integers(-3, 103, (len(seq), kv, n)).astype(np.int32)
    lists[2] = -1
    lists[5, :, 1:] = 5
    lists[0, 0, [0, n // 2, n - 1]] = [2 ** 31 - 1, -2 ** 31, 99]
    lt = torch.from_numpy(lists).cuda()
    q = sc.random(len(seq), sc.hq, d)
    lse = sc.attend(batch, q, lt)[1]
    prev = torch.rand(len(lens), kv, sc.max_pages, device="cuda")
    for workspace in (True, False):
        got = P.run_weigh(sc, batch, q, lse, prev, lt, workspace=workspace)
        P.check_weigh(sc, q, lse, got, prev, lt)
        assert torch.equal(got, P.run_weigh(sc, batch, q, lse, prev.clone(), lt, alias=True, workspace=workspace))
