"""The forms that the calls on drafted tokens take by size -- row blocks and partitions of the attention, shared slots whose users are split for the
weights --, and the loop of examples/draft_decode.py, against the float64 reference.  Bounds: those of test_gpu_draft.py, from which the checks come."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import draft_ref as ref

from gpu_util import DEV, bf16, host
from test_gpu_draft import check_attention, make, random_tree, stored

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))

pytestmark = pytest.mark.gpu


def trees(seed, Hq, Hkv, D, T, formats, lengths, C):
    B, n_c = len(lengths), len(lengths[0])
    pc, g, kv = make(seed, Hq, Hkv, D, C, formats, [C] * (B * n_c), max_pos=16384)
    q, k, v = bf16(1.5 * g.standard_normal((B, Hq, T, D))), bf16(g.standard_normal((B, Hkv, T, D))), bf16(g.standard_normal((B, Hkv, T, D)))
    return pc, kv, q, k, v, np.arange(B * n_c).reshape(B, n_c), np.array(lengths, np.int32), [random_tree(g, T, T - b) for b in range(B)]


# rows of a kv head (heads of it x nodes) on both sides of every block: the decode kernel ends at 32, blocks of 64, 128 and 192 rows behind it
@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [16, 17, 32, 33, 64, 65, 96, 97, 128, 129])
def test_rows_around_the_blocks(T, D, formats):
    pc, kv, q, k, v, ids, used, parents = trees(21 + T, 2, 1, D, T, formats, [[100, 64, 3], [0, 31, 33]], 128)
    check_attention(pc, kv, q, k, v, ids, used, parents)
    pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("Hq,T,D", [(2, 20, 128), (2, 50, 128), (3, 60, 128), (2, 100, 64), (2, 20, 64), (4, 60, 64)])
def test_partitions_of_every_block(Hq, T, D, formats):
    """More partitions than tiles among them, so that some have nothing; a query without a cached key."""
    pc, kv, q, k, v, ids, used, parents = trees(22, Hq, 1, D, T, formats, [[256, 65, 200], [0, 0, 0], [1, 0, 255]], 256)
    for n in (1, 2, 5, 9, 13):
        check_attention(pc, kv, q, k, v, ids, used, parents, n_splits=n)
    pc.close()


def test_a_call_of_many_rows_merges_heads_together():
    """More than 20 rows a CU with few partitions: two, three and four heads of a group in one wavefront of the merge."""
    for Hq, Hkv in ((8, 4), (12, 4), (16, 4), (28, 4)):
        pc, kv, q, k, v, ids, used, parents = trees(23, Hq, Hkv, 64, 100, "bf16", [[70]] * (60 * 100 // (Hq * 100) + 8), 128)
        out, lse = pc.percache_attention_draft(0, q, k, v, slot_ids=ids, used_len=used, parents=parents, lse_out=True)
        one = [pc.percache_attention_draft(0, q[b:b + 1].contiguous(), k[b:b + 1].contiguous(), v[b:b + 1].contiguous(), slot_ids=ids[b:b + 1], used_len=used[b:b + 1],
                                           parents=parents[b:b + 1], lse_out=True) for b in (0, len(parents) - 1)]
        torch.cuda.synchronize()
        for b, (o, l) in zip((0, len(parents) - 1), one):
            assert torch.allclose(out[b].float(), o[0].float(), atol=2.0 ** -6, rtol=2.0 ** -6) and torch.allclose(lse[b], l[0], atol=1e-4, rtol=0)
        pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("Hq,Hkv,D,B,T,C", [(2, 2, 64, 40, 1, 1024), (4, 2, 128, 13, 3, 128), (6, 2, 64, 9, 33, 128), (2, 1, 128, 5, 70, 192)])
def test_weights_of_slots_that_many_queries_share(Hq, Hkv, D, B, T, C, formats):
    """Two slots named by every query, to lengths of their own; one of its own each.  (In the first shape the workspace has room for one slot's split only.)"""
    pc, g, kv = make(24, Hq, Hkv, D, C, formats, [C - 5, C] + [40] * B, max_pos=16384)
    ids = np.array([[0, 2 + b, 1] for b in range(B)])
    used = np.array([[C - 5 - 2 * b, 40, C if b else 0] for b in range(B)], np.int32)
    q, k, v = bf16(2 * g.standard_normal((B, Hq, T, D))), bf16(g.standard_normal((B, Hkv, T, D))), bf16(g.standard_normal((B, Hkv, T, D)))
    parents = [random_tree(g, T) for _ in range(B)]
    lse, found = check_attention(pc, kv, q, k, v, ids, used, parents)
    start = torch.rand((2 + B, Hkv, C), device=DEV)
    out = start.clone()
    draft = pc.percache_attention_weights(0, q, k, lse, start, out, slot_ids=ids, used_len=used, parents=parents)
    again = start.clone()
    draft2 = pc.percache_attention_weights(0, q, k, lse, again, again, slot_ids=ids, used_len=used, parents=parents)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(draft, draft2)
    want, paid, rel = start.double().cpu().numpy(), np.zeros((2 + B, Hkv, C)), 0.0
    for b in range(B):
        wl_, S, keys, probs = found[b]
        c, d = ref.weights(probs, Hq, Hkv, T, keys - T, range(T))
        lo = 0
        for s, u in zip(ids[b], used[b]):
            paid[s, :, :u] += c[:, lo:lo + u]
            lo += u
        live = np.isfinite(wl_)
        rel = max(rel, (D * S + keys + 16 * np.abs(wl_[live]).max(initial=0) + 128 + B * Hq // Hkv * T) * 2.0 ** -24)
        assert (np.abs(draft[b].double().cpu().numpy() - d) <= rel * d).all()
    got = out.double().cpu().numpy()
    assert (np.abs(got - want - paid) <= rel * paid + 2.0 ** -23 * (want + paid)).all()
    assert np.array_equal(got[paid == 0], want[paid == 0])
    pc.close()


@pytest.mark.parametrize("n8", [0, 2, 5])
def test_decoding_by_drafts_over_a_bounded_cache(n8):
    """Every step's attention against the reference over what the slots hold, what a cut slot holds against the tokens that it must have kept."""
    import draft_decode
    d = draft_decode.DraftDecoder(batch=2, nodes=12, chunks=3, capacity=128, budget=70, hidden=256, heads=4, kv_heads=2, head_dim=64, first=2, last=9, seed=3, n_slots_8bit=n8)
    cuts = 0
    for step in range(60):
        before, held, w = stored(d.pc), d.held.copy(), d.weights.clone()
        r = d.step()
        after = stored(d.pc)
        for b in range(2):
            own = d.chunks + b
            assert d.pc.percache_kv_len(0, own) == d.held[b] <= d.capacity - d.nodes
            if step % 20 == 19 or len(r["cut"]):
                kc, vc = (np.concatenate([before[s][x] for s in (0, 1, 2, own)], 1) for x in (0, 1))
                want, lse, size, S, probs = ref.attend(*(host(r[n][b]).astype(np.float64) for n in ("q",)), kc, vc, *(host(r[n][b]).astype(np.float64) for n in ("k", "v")),
                                                       ref.ancestors(r["parents"][b].tolist()))
                got = host(r["out"][b]).astype(np.float64).reshape(want.shape)
                assert (np.abs(got - want) <= (2.0 ** -7 + 2.0 ** -13) * size).all()
            n = held[b] + r["n_path"][b]
            if b not in r["cut"]:
                # the path behind what the slot held (codes of the block that was open are made afresh)
                whole = held[b] if own < d.pc.cfg.n_slots - n8 else held[b] // 64 * 64
                assert all(np.array_equal(after[own][x][:, :whole], before[own][x][:, :whole]) for x in (0, 1))
                if own < d.pc.cfg.n_slots - n8:
                    for x, name in ((0, "k"), (1, "v")):
                        assert np.array_equal(after[own][x][:, held[b]:n], host(r[name][b]).astype(np.float64)[:, r["path"][b, :r["n_path"][b]]])
            else:
                cuts += 1
                assert d.held[b] == min(n, 70)
                if own < d.pc.cfg.n_slots - n8:   # the first and the last tokens are among the kept ones
                    path_k = host(r["k"][b]).astype(np.float64)[:, r["path"][b, :r["n_path"][b]]]
                    full = np.concatenate([before[own][0], path_k], 1)
                    assert np.array_equal(after[own][0][:, :2], full[:, :2]) and np.array_equal(after[own][0][:, -9:], full[:, -9:])
        assert torch.isfinite(d.weights).all() and (d.weights[:3] >= w[:3]).all()
    # every accepted row's probabilities sum to one: what the shared chunks and the slots were paid is at most the rows' number
    assert cuts >= 2
    d.close()
