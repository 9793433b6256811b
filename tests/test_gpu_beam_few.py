"""examples/beam_decode.py with fewer continuations than beams, on the device."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))

pytestmark = pytest.mark.gpu


def test_three_tokens_and_four_beams():
    import beam_decode
    d = beam_decode.BeamDecoder(batch=2, beams=4, chunks=1, capacity=128, longest=20, vocab=3, hidden=256, heads=4, kv_heads=2, seed=9)
    d.prompts()
    torch.cuda.synchronize()
    assert (d.parent == [[0, 0, 0, -1]] * 2).all() and (d.tokens[:, 3] == -1).all() and (d.scores[:, 3] == -float("inf")).all()
    assert [sorted(t[:3, 0]) for t in d.tokens] == [[0, 1, 2]] * 2
    assert [d.pc.percache_kv_len(0, int(s)) for s in d.slots.ravel()] == [int(n) for n in np.repeat(d.lengths, 4)]
    for step in range(3):
        d.step()
        torch.cuda.synchronize()
        assert (d.parent >= 0).all() and (d.tokens >= 0).all() and torch.isfinite(d.scores).all()
        assert step or not (d.parent == 3).any()
        assert all(len({tuple(t) for t in of_request}) == 4 for of_request in d.tokens)
        assert (d.scores[:, :-1] >= d.scores[:, 1:]).all()
    d.close()
