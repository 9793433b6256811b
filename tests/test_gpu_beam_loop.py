"""The loop of examples/beam_decode.py: prompts packed, kept, handed to beams, extended token by token.  Every call is checked against the float64
reference of its kind, and every beam's slot against the rows of the tokens that it goes back to, bit for bit."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import kv_fp8
from oracle import packed_ref as ref

from gpu_util import host
from test_gpu_draft import cached, stored

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))

pytestmark = pytest.mark.gpu


def check_attention(d, kv):
    """The last layer call against the reference (bounds: test_gpu_packed.py); kv: the slots' contents at the call."""
    L = d.last
    q, k, v = (host(L[x]).astype(np.float64) for x in "qkv")
    out = host(L["out"]).astype(np.float64).reshape(q.shape[1], d.heads, d.D)
    for s in range(len(L["start"]) - 1):
        a, b = int(L["start"][s]), int(L["start"][s + 1])
        kc, vc = cached(kv, L["ids"][s], [kv[i][0].shape[1] for i in L["ids"][s]])
        want, _, size, _ = ref.attend(q[:, a:b], k[:, a:b], v[:, a:b], kc, vc)
        assert (np.abs(out[a:b] - want) <= (2.0 ** -7 + 2.0 ** -13) * size).all(), s


@pytest.mark.parametrize("D,heads,kv_heads,n8", [(128, 4, 2, 0), (64, 6, 2, 0), (64, 4, 1, 12)])
def test_beams_of_prompts_of_different_lengths(D, heads, kv_heads, n8):
    import beam_decode
    B, K = 3, 4
    d = beam_decode.BeamDecoder(batch=B, beams=K, chunks=2, capacity=128, longest=100, vocab=999, hidden=256, heads=heads, kv_heads=kv_heads, head_dim=D, seed=5,
                                n_slots_8bit=n8)
    pc, choose = d.pc, d.choose
    rows = {}          # slot -> (k, v) rows that it has to hold
    kept = lambda x: kv_fp8.round_trip(x) if n8 else x

    def checked_choose(logits):
        scores = d.scores.clone()
        choose(logits)
        torch.cuda.synchronize()
        parent, token, score = ref.beams(logits.double().cpu().numpy(), scores.double().cpu().numpy(), K)
        assert np.array_equal(d.parent, parent) and np.array_equal(d.token, token)
        assert (np.abs(d.scores.double().cpu().numpy() - score) <= 2.0 ** -21 + 2.0 ** -23 * np.abs(score)).all()
    d.choose = checked_choose

    def check_slots():
        got = stored(pc)
        for s, want in rows.items():
            assert all(np.array_equal(got[s][x], want[x]) for x in (0, 1)), s

    before = stored(pc)
    d.prompts()
    check_attention(d, before)
    for b in range(B):
        a, e = int(d.last["start"][b]), int(d.last["start"][b + 1])
        for i in range(K):
            rows[int(d.slots[b, i])] = tuple(kept(host(d.last[x][:, a:e]).astype(np.float64)) for x in "kv")
    check_slots()
    for _ in range(12):
        before = stored(pc)
        d.step()
        check_attention(d, before)
        new = [tuple(host(d.last[x][:, r:r + 1]).astype(np.float64) for x in "kv") for r in range(B * K)]
        grown = {}
        for r, s in enumerate(d.slots.ravel()):
            full = tuple(np.concatenate([rows[int(s)][x], new[r][x]], 1) for x in (0, 1))
            lo = (full[0].shape[1] - 1) // 64 * 64      # (an 8-bit slot quantises the block of the new token afresh)
            grown[int(s)] = tuple(np.concatenate([x[:, :lo], kept(x[:, lo:])], 1) for x in full)
        for b in range(B):
            for i in range(K):
                rows[int(d.slots[b, i])] = grown[int(d.slots[b, d.parent[b, i]])]
        check_slots()
    assert d.tokens.shape == (B, K, 13) and len({tuple(t) for t in d.tokens[0]}) == K
    d.close()
