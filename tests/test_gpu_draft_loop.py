"""The loop of examples/draft_decode.py, call by call: what each append and each cut leaves in the queries' own slots of either format, exactly, and what
a step's accepted rows pay in all."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import draft_ref as ref
from oracle import kv_fp8

from gpu_util import host
from test_gpu_draft import stored

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n8", [0, 1, 2, 5])
def test_what_every_call_of_the_loop_leaves(n8):
    import draft_decode
    d = draft_decode.DraftDecoder(batch=2, nodes=12, chunks=3, capacity=128, budget=70, hidden=256, heads=4, kv_heads=2, head_dim=64, first=2, last=9, seed=4, n_slots_8bit=n8)
    pc, n16, done = d.pc, d.pc.cfg.n_slots - n8, dict(weights=0, append=0, cuts=0)
    weights, append, keep = pc.percache_attention_weights, pc.percache_kv_append_path, pc.percache_kv_keep

    def check_weights(layer, q, k, lse, w_in, w_out, *, path, n_path, **kw):
        before, kv = w_in.double(), stored(pc)
        paid = weights(layer, q, k, lse, w_in, w_out, path=path, n_path=n_path, **kw)
        torch.cuda.synchronize()
        # every accepted row's probabilities sum to one, for each of the two heads of a group
        total = (w_out.double() - before).sum((0, 2)) + paid.double().sum((0, 2))
        longest = max(float(np.linalg.norm(x, axis=-1).max(initial=0)) for x, _ in kv)
        S = float(q.double().norm(dim=-1).max()) * max(longest, float(k.double().norm(dim=-1).max())) / 8   # (sum |q_d k_d| <= |q| |k|; sqrt(D) = 8)
        rows, n = 2 * int(np.sum(n_path)), 3 * 128 + 128 + 12
        rel = (64 * S + n + 16 * float(lse.abs().max()) + 128 + rows) * 2.0 ** -24
        assert ((total - rows).abs() <= rel * rows + 2.0 ** -23 * w_out.double().sum((0, 2))).all(), (total, rows)
        done["weights"] += 1
        return paid

    def check_append(layer, k, v, slots, path, *, n_path, weights, draft_weights):
        before, w = stored(pc), weights.clone()
        append(layer, k, v, slots, path, n_path=n_path, weights=weights, draft_weights=draft_weights)
        torch.cuda.synchronize()
        after = stored(pc)
        for b, s in enumerate(slots):
            at, held = path[b, :n_path[b]], before[s][0].shape[1]
            for x, new in ((0, k), (1, v)):
                full = np.concatenate([before[s][x], host(new[b]).astype(np.float64)[:, at]], 1)
                lo = held // 64 * 64
                if s >= n16:
                    full[:, lo:] = kv_fp8.round_trip(full[:, lo:])
                assert np.array_equal(after[s][x], full), (s, x)
            w[s, :, held:held + len(at)] = draft_weights[b][:, torch.as_tensor(at.astype(np.int64), device=w.device)]
        assert torch.equal(weights, w)
        assert all(np.array_equal(after[s][x], before[s][x]) for s in range(3) for x in (0, 1))
        done["append"] += 1

    def check_keep(layer, slots, budget, weights, *, n_first, n_last):
        before, w = stored(pc), weights.cpu().numpy().astype(np.float64)
        idx = keep(layer, slots, budget, weights, n_first=n_first, n_last=n_last)
        torch.cuda.synchronize()
        after = stored(pc)
        for z, s in enumerate(slots):
            rows = [ref.keep(w[s, h], before[s][0].shape[1], budget, n_first, n_last) for h in range(2)]
            assert idx[z].cpu().tolist() == rows
            for x in (0, 1):
                want = np.stack([before[s][x][h][rows[h]] for h in range(2)])
                assert np.array_equal(after[s][x], kv_fp8.round_trip(want) if s >= n16 else want), (s, x)
            assert all(np.array_equal(weights[s, h, :budget].cpu().numpy(), w[s, h, rows[h]]) for h in range(2))
            done["cuts"] += 1
        return idx

    pc.percache_attention_weights, pc.percache_kv_append_path, pc.percache_kv_keep = check_weights, check_append, check_keep
    for _ in range(60):
        d.step()
    assert done["weights"] == done["append"] == 60 and done["cuts"] >= 2
    d.close()
