"""The host side of examples/beam_decode.py: beams that do not exist, positions behind the chunks."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import packed_ref as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
import beam_decode  # noqa: E402


class Library:
    """The selection by the reference; copies are written down."""
    def __init__(self):
        self.copies = []

    def percache_beam_select(self, logits, scores, best):
        p, t, s = ref.beams(logits.double().numpy(), scores.double().numpy(), best)
        return torch.from_numpy(p.astype(np.int32)), torch.from_numpy(t.astype(np.int32)), torch.from_numpy(s.astype(np.float32))

    def percache_kv_fork(self, src, dst):
        self.copies.append((list(map(int, src)), list(map(int, dst))))


def decoder(batch, beams, chunks, vocab):
    d = beam_decode.BeamDecoder.__new__(beam_decode.BeamDecoder)
    d.batch, d.beams, d.chunks, d.vocab, d.pc = batch, beams, chunks, vocab, Library()
    d.slots = chunks + np.arange(batch * beams, dtype=np.int32).reshape(batch, beams)
    d.scores, d.tokens = torch.zeros((batch, 1)), np.zeros((batch, beams, 0), np.int64)
    return d


def test_fewer_continuations_than_beams():
    d = decoder(2, 4, 1, 3)
    x = torch.tensor([[[0.0, 2.0, 1.0]], [[-np.inf, 5.0, -np.inf]]])
    d.choose(x)
    assert d.tokens[:, :, 0].tolist() == [[1, 2, 0, -1], [1, -1, -1, -1]]
    assert d.parent.tolist() == [[0, 0, 0, -1], [0, -1, -1, -1]] and torch.isinf(d.scores).tolist() == [[False] * 3 + [True], [False] + [True] * 3]
    assert d.pc.copies[-1] == ([1] * 4 + [5] * 4, [1, 2, 3, 4, 5, 6, 7, 8])     # the slot that the beams open with
    # the next step goes on from beams that exist only; a request without any continuation keeps its slots filled
    x = torch.zeros((2, 4, 3))
    x[0, 3] = 100.0
    x[1, 0] = float("nan")
    d.choose(x)
    assert (d.parent[0] >= 0).all() and 3 not in d.parent[0] and (d.parent[1] == -1).all()
    assert all(t[0] == [1, 2, 0][p] for t, p in zip(d.tokens[0].tolist(), d.parent[0])) and (d.tokens[1] == -1).all()
    assert d.pc.copies[-1][0][4:] == [5] * 4


@pytest.mark.parametrize("capacity", [64, 512, 4096])
def test_prompts_start_behind_the_chunks(capacity):
    d = decoder(1, 2, 3, 10)
    d.capacity, d.lengths, d.position, d.rng = capacity, np.array([50]), np.zeros(1, np.int64), np.random.default_rng(1)
    pos = d.prompt_positions(0)
    assert pos.shape == (3, 50) and pos.min() == 3 * capacity and d.position[0] == pos.max() + 1 and pos.max() < 4 * capacity
