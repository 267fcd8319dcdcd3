"""The buffers of TokenPipeline, on the host: which are kept, which refused."""

from __future__ import annotations

import types
import weakref

import pytest
import torch

from paper_2606_30709_amd import hga
from paper_2606_30709_amd.pipeline import TokenPipeline


@pytest.fixture
def pipe(monkeypatch):
    state = types.SimpleNamespace(capturing=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state.capturing)
    pool = types.SimpleNamespace(device=torch.device("cpu"))
    p = TokenPipeline(types.SimpleNamespace(plan=None, pool=pool))
    p.state = state
    return p


def test_what_a_capture_used_outlives_larger_steps(pipe):
    small = pipe._buffer("out", (2, 8), torch.float32).data_ptr()
    pipe.state.capturing = True
    assert pipe._buffer("out", (2, 8), torch.float32).data_ptr() == small
    held = weakref.ref(pipe._buf["out"])
    pipe.state.capturing = False
    large = pipe._buffer("out", (64, 8), torch.float32)
    assert large.data_ptr() != small and held() is not None and held().data_ptr() == small
    # one that no capture used is given back
    free = weakref.ref(pipe._buf["out"])
    del large
    assert pipe._buffer("out", (2, 8), torch.float32).data_ptr() == free().data_ptr()
    pipe._buffer("out", (128, 8), torch.float32)
    assert free() is None and held() is not None


def test_a_captured_step_allocates_nothing(pipe):
    pipe._buffer("lists", (4,), torch.int32)
    pipe.state.capturing = True
    pipe._buffer("lists", (3,), torch.int32)
    for name, n in (("lists", 5), ("attend", 1)):
        with pytest.raises(hga.HgaError) as e:
            pipe._buffer(name, (n,), torch.int32)
        assert e.value.status == -1
    assert "attend" not in pipe._buf and pipe._buf["lists"].numel() == 4
