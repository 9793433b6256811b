"""What the binding keeps from call to call, without a device: its calls reach a stand-in for the library that does nothing."""
import weakref

import numpy as np
import pytest
import torch

from paper_2601_11553_amd.binding import Config, Percache


class Library:
    """Sizes are the sums of their arguments; every other call is fine."""
    def __getattr__(self, name):
        return lambda ctx, *args: sum(args) if name.endswith("_bytes") else 0


@pytest.fixture
def pc(monkeypatch):
    """A context whose tensors are on the CPU."""
    pc = Percache.__new__(Percache)
    pc.lib, pc.ctx, pc.device = Library(), None, torch.device("cpu")
    pc.cfg = Config(1, 256, 4, 2, 64, 8, 64, 1000, 1e4, 0, 0, 0, 0)
    pc._draft_ws, pc._draft_bytes, pc._all_chunks = {}, {}, {}
    monkeypatch.setattr(pc, "_raw_stream", lambda: 5, raising=False)
    monkeypatch.setattr(pc, "_want", lambda *a: None, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
    return pc


def test_ever_new_shapes_are_not_kept_for_good(pc):
    for n in range(1, 3000):
        assert pc._draft_need(2, n, 3) == n + 5
        (_, _, nc), _, _, nc_p, max_chunks = pc._draft_chunks(n, np.zeros((n, 2), np.int32), None, None)
        assert max_chunks == 2 and nc.size == n and (nc == 2).all() and nc_p == nc.ctypes.data
        assert pc._draft_need(2, n, 3) == n + 5
        assert len(pc._draft_bytes) <= Percache.kept_shapes and len(pc._all_chunks) <= Percache.kept_shapes


def test_calls_on_packed_rows_keep_no_size_for_good(pc):
    for n in range(1, 2000):
        x = torch.empty((4, n, 64), dtype=torch.bfloat16)
        pc.percache_attention_packed(0, x, x[:2], x[:2], [0, n])
        assert len(pc._draft_bytes) <= Percache.kept_shapes
    assert ("packed", 1, n, 0) in pc._draft_bytes


def test_a_captured_calls_workspace_is_its_graphs(pc, monkeypatch):
    """Neither the stream's own one, which eager calls and other graphs would write, nor kept behind the call."""
    made, given, empty = [], [], torch.empty

    def watched(n, **kw):
        t = empty(n, **kw)
        made.append((weakref.ref(t), t.data_ptr(), n))
        return t
    monkeypatch.setattr(torch, "empty", watched)
    monkeypatch.setattr(Library, "percache_beam_select", lambda lib, ctx, *args: given.append(args[-3]) or 0, raising=False)
    x, scores = torch.zeros((2, 3, 40)), torch.zeros((2, 3))
    logits = type("OnTheGpu", (), dict(dim=lambda s: 3, dtype=torch.float32, is_cuda=True, stride=lambda s, i: x.stride(i), shape=x.shape, data_ptr=lambda s: 0))()
    call = lambda: pc.percache_beam_select(logits, scores, 4)
    inside = lambda at, ws: ws[1] <= at < ws[1] + ws[2]
    call()
    own = pc._draft_ws[5]
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: True)
    for _ in range(2):
        call()
    monkeypatch.setattr(torch._C, "_cuda_isCurrentStreamCapturing", lambda: False)
    call()
    assert len(made) == 3 and len(given) == 4
    assert inside(given[0], made[0]) and inside(given[1], made[1]) and inside(given[2], made[2]) and inside(given[3], made[0])
    assert made[0][0]() is own and pc._draft_ws == {5: own} and made[1][0]() is None and made[2][0]() is None
