"""Eviction inside a slot through the C ABI against the float64 reference (oracle/draft_ref.keep).  Everything here is selection and copies: exact."""
import numpy as np
import pytest
import torch

from oracle import draft_ref as ref
from oracle import kv_fp8

from gpu_util import DEV, bf16, host
from test_gpu_draft import make, random_tree, stored

pytestmark = pytest.mark.gpu


def check(pc, before, weights, slots, keep, n_first, n_last, dst=None, layer=0):
    Hkv, C = pc.cfg.n_kv_heads, pc.cfg.slot_capacity
    w = torch.from_numpy(weights).to(DEV)
    want_w = weights.copy()
    idx = pc.percache_kv_keep(layer, slots, keep, w, n_first=n_first, n_last=n_last, dst_slots=dst).cpu().numpy()
    torch.cuda.synchronize()
    keeps = np.broadcast_to(keep, (len(slots),))
    to = slots if dst is None else dst
    n16 = pc.cfg.n_slots - pc.cfg.n_slots_8bit
    assert idx.shape == (len(slots), Hkv, keeps.max())
    after = stored(pc, layer)
    for z, (s, d) in enumerate(zip(slots, to)):
        have = before[s][0].shape[1]
        n = min(int(keeps[z]), have)
        assert pc.percache_kv_len(layer, d) == n
        rows = []
        for h in range(Hkv):
            r = ref.keep(weights[s, h].astype(np.float64), have, int(keeps[z]), n_first, n_last)
            assert idx[z, h, :n].tolist() == r and (idx[z, h, n:] == -1).all(), (z, h)
            rows.append(r)
            want_w[d, h, :n] = weights[s, h, r]
        for x in (0, 1):
            want = np.stack([before[s][x][h][rows[h]] for h in range(Hkv)])
            assert np.array_equal(after[d][x], kv_fp8.round_trip(want) if d >= n16 else want), (z, x)
    named = set(to)
    for s in range(pc.cfg.n_slots):
        if s not in named:
            assert all(np.array_equal(after[s][x], before[s][x]) for x in (0, 1))
    got = w.cpu().numpy()
    for z, d in enumerate(to):   # (behind the kept ones the weights are of no meaning)
        n = after[d][0].shape[1]
        assert np.array_equal(got[d, :, :n], want_w[d, :, :n], equal_nan=True)
        got[d, :, n:] = want_w[d, :, n:] = 0
    assert np.array_equal(got, want_w, equal_nan=True)
    return after


def weights_of(g, kind, shape):
    w = g.random(shape).astype(np.float32)
    if kind == "heavy":
        w = (-np.log(w)) ** 3 * np.float32(1e-3)
    elif kind == "ties":
        w = np.floor(w * 3)
    elif kind == "equal":
        w[:] = 0.0
    elif kind == "odd":   # negative ones, both zeros, infinities, NaN, subnormals
        special = np.array([-1.5, 0.0, -0.0, np.inf, -np.inf, np.nan, 1e-42, -1e-42, 3e38, 1.0], np.float32)
        w = special[g.integers(0, len(special), shape)]
    return w.astype(np.float32)


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "odd"])
@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("Hkv,D,C,lengths,keep,n_first,n_last", [
    (2, 64, 64, [64, 1, 33, 64], [1, 1, 32, 63], 0, 0), (2, 128, 192, [192, 65, 128, 100], 64, 4, 16), (1, 128, 320, [320, 257], [65, 129], 1, 0),
    (8, 128, 512, [512, 300], [256, 299], 4, 32), (2, 64, 1088, [1088, 1000, 70], [500, 999, 70], 0, 64), (4, 128, 64, [10, 20], [30, 20], 3, 5)])
def test_kept_tokens_in_place(Hkv, D, C, lengths, keep, n_first, n_last, formats, kind):
    pc, g, before = make(20, 2 * Hkv, Hkv, D, C, formats, lengths + [5])
    check(pc, before, weights_of(g, kind, (len(lengths) + 1, Hkv, C)), list(range(len(lengths))), keep, n_first, n_last)
    pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("D", [64, 128])
def test_kept_tokens_into_other_slots_of_either_format(formats, D):
    lengths = [130, 0, 192, 64, 100, 0, 77, 0]
    pc, g, before = make(21, 4, 2, D, 192, formats, lengths)
    # some to empty slots, one over a slot that held something, one in place; in a mixed store also across the formats
    check(pc, before, weights_of(g, "heavy", (8, 2, 192)), [0, 4, 2, 6], [100, 64, 129, 70], 2, 7, dst=[5, 1, 3, 6])
    pc.close()


def test_more_slots_than_one_launch_takes():
    n = 150
    pc, g, before = make(22, 2, 1, 64, 128, "mixed", [128 - i % 50 for i in range(n)])
    order = g.permutation(n)[:140].tolist()
    check(pc, before, weights_of(g, "heavy", (n, 1, 128)), order, [int(x) for x in g.integers(8, 129, 140)], 3, 4)
    pc.close()


def test_the_same_call_again_changes_nothing():
    pc, g, before = make(23, 4, 2, 128, 256, "mixed", [256, 256])
    w = weights_of(g, "heavy", (2, 2, 256))
    after = check(pc, before, w, [0, 1], 100, 4, 8)
    wd = torch.from_numpy(w).to(DEV)
    idx = pc.percache_kv_keep(0, [0, 1], 100, wd, n_first=4, n_last=8)
    torch.cuda.synchronize()
    assert (idx == torch.arange(100, dtype=torch.int32, device=DEV)).all()
    assert all(np.array_equal(a[x], b[x]) for a, b in zip(stored(pc), after) for x in (0, 1))
    pc.close()


def test_a_layer_of_its_own():
    """Only the named layer changes, its slots in both formats."""
    pc, g, kv1 = make(24, 2, 1, 64, 64, "mixed", [64, 64], n_layers=2)
    for s in range(2):
        pc.percache_kv_put(0, s, bf16(g.standard_normal((1, 60, 64))), bf16(g.standard_normal((1, 60, 64))))
    first = stored(pc, 0)
    check(pc, kv1, weights_of(g, "heavy", (2, 1, 64)), [0, 1], 30, 1, 1, layer=1)
    assert all(np.array_equal(a[x], b[x]) for a, b in zip(stored(pc, 0), first) for x in (0, 1))
    pc.close()


def test_decoding_on_over_what_was_kept():
    """The whole round: a tree verified over the cache, the accepted path appended with its weights, the slot cut, the next tree over it -- against the
    reference that does the same on lists of rows."""
    Hq, Hkv, D, T = 4, 2, 128, 9
    pc, g, kv = make(25, Hq, Hkv, D, 128, "bf16", [100])
    rows = [(kv[0][0][h], kv[0][1][h]) for h in range(Hkv)]     # per head: keys, values
    w_ref = np.zeros((Hkv, 128))
    w = torch.zeros((1, Hkv, 128), device=DEV)
    have = 100
    for step in range(4):
        q, k, v = bf16(2 * g.standard_normal((1, Hq, T, D))), bf16(g.standard_normal((1, Hkv, T, D))), bf16(g.standard_normal((1, Hkv, T, D)))
        parents = random_tree(g, T)
        out, lse = pc.percache_attention_draft(0, q, k, v, slot_ids=[[0]], parents=[parents], lse_out=True)
        path = [T - 1]
        while parents[path[0]] >= 0:
            path.insert(0, parents[path[0]])
        dw = pc.percache_attention_weights(0, q, k, lse, w, w, slot_ids=[[0]], parents=[parents], path=[path])
        pc.percache_kv_append_path(0, k, v, [0], [path], weights=w, draft_weights=dw)
        want, _, size, _, probs = ref.attend(*(host(x[0]).astype(np.float64) for x in (q,)), np.stack([r[0] for r in rows]), np.stack([r[1] for r in rows]),
                                             host(k[0]).astype(np.float64), host(v[0]).astype(np.float64), ref.ancestors(parents))
        torch.cuda.synchronize()
        got = host(out[0]).astype(np.float64).reshape(T, Hq, D)
        assert (np.abs(got - want) <= (2.0 ** -7 + 2.0 ** -13) * size).all()
        c, d = ref.weights(probs, Hq, Hkv, T, have, path)
        w_ref[:, :have] += c
        w_ref[:, have:have + len(path)] = d[:, path]
        rows = [(np.concatenate([r[0], host(k[0, h, path])]), np.concatenate([r[1], host(v[0, h, path])])) for h, r in enumerate(rows)]
        have += len(path)
        assert np.allclose(w[0, :, :have].cpu().numpy(), w_ref[:, :have], rtol=1e-4, atol=1e-9)
        idx = pc.percache_kv_keep(0, [0], 90, w, n_first=4, n_last=10)[0].cpu().numpy()
        n = min(90, have)
        # (the library's own sums decide: they differ from the reference's by rounding; the choice agrees where the weights are not that close)
        for h in range(Hkv):
            mine = ref.keep(w_ref[h], have, 90, 4, 10)
            for a in set(idx[h, :n].tolist()) ^ set(mine):
                cut = np.sort(w_ref[h, 4:have - 10])[::-1][n - 15]
                assert abs(w_ref[h, a] - cut) < 1e-4 * cut
            w_ref[h, :n] = w_ref[h, idx[h, :n]]
        rows = [(r[0][idx[h, :n]], r[1][idx[h, :n]]) for h, r in enumerate(rows)]
        have = n
    pc.close()
