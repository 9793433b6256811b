"""Calls on drafted tokens at the edges of their lists and numbers, against the float64 reference.  Bounds: those of test_gpu_draft.py."""
import numpy as np
import pytest
import torch

from oracle import draft_ref as ref
from oracle import kv_fp8

from gpu_util import DEV, bf16, host
from test_gpu_draft import cached, make, random_tree, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,T,live,skipped", [(64, 2000, 1, 2000), (128, 1000, 1, 834), (64, 300, 40, 300)])
@pytest.mark.parametrize("formats", ["bf16", "8bit"])
def test_a_skipped_query_with_a_longer_path_than_any_other(D, T, live, skipped, formats):
    """The skipped query first, in the middle and last; what the others append is what they append without it."""
    pc, g, kv = make(31, 2, 2, D, 64, formats, [10, 0])
    k, v = bf16(g.standard_normal((4, 2, T, D))), bf16(g.standard_normal((4, 2, T, D)))
    path = g.integers(0, T, (4, skipped))
    want = {}
    for slots in ([0, 1, -1, -1], [-1, 0, -7, 1], [-1, -1, 0, 1], [0, -1, 1, -1]):
        n_path = [live if s >= 0 else skipped for s in slots]
        pc.percache_kv_put(0, 0, *(bf16(x) for x in kv[0]))
        pc.percache_kv_evict(0, 1)
        pc.percache_kv_append_path(0, k, v, slots, path, n_path=n_path)
        got = stored(pc)
        for s in (0, 1):
            b = slots.index(s)
            pc.percache_kv_put(0, 0, *(bf16(x) for x in kv[0]))
            pc.percache_kv_evict(0, 1)
            pc.percache_kv_append_path(0, k[b:b + 1].contiguous(), v[b:b + 1].contiguous(), [s], path[b:b + 1, :live])
            alone = stored(pc)[s]
            assert got[s][0].shape[1] == (10 if s == 0 else 0) + live
            assert all(np.array_equal(got[s][x], alone[x]) for x in (0, 1))
            new = host(k[b][:, path[b, :live]]).astype(np.float64)
            if formats == "bf16":
                assert np.array_equal(got[s][0][:, -live:], new)
    pc.close()


def test_a_skipped_query_behind_a_full_list():
    """207 queries with one node each and a skipped one with 200: the last record of the launch."""
    pc, g, kv = make(32, 2, 1, 64, 64, "bf16", [0] * 207)
    k, v = bf16(g.standard_normal((208, 1, 256, 64))), bf16(g.standard_normal((208, 1, 256, 64)))
    path = g.integers(0, 256, (208, 200))
    pc.percache_kv_append_path(0, k, v, list(range(207)) + [-1], path, n_path=[1] * 207 + [200])
    torch.cuda.synchronize()
    for s in (0, 100, 206):
        got = pc.percache_kv_get(0, s)
        assert torch.equal(got[0][:, 0], k[s, :, path[s, 0]]) and torch.equal(got[1][:, 0], v[s, :, path[s, 0]])
    assert all(pc.percache_kv_len(0, s) == 1 for s in range(207))
    pc.close()


# rows of a kv head up to 32 (one kernel with the nodes), above, and so many that heads are merged together
@pytest.mark.parametrize("Hq,Hkv,D,T,B", [(4, 2, 128, 7, 1), (4, 2, 64, 16, 2), (6, 2, 128, 20, 2), (8, 2, 64, 30, 1), (2, 1, 128, 200, 1), (16, 4, 64, 70, 8)])
@pytest.mark.parametrize("formats,n_splits", [("bf16", 0), ("bf16", 1), ("bf16", 2), ("bf16", 5), ("8bit", 0), ("mixed", 3)])
def test_infinite_values_that_a_row_sees(Hq, Hkv, D, T, B, formats, n_splits):
    """V of a cached key (bf16 slots) and of nodes infinite in some dimensions: infinite there, NaN where both signs meet, and the usual numbers elsewhere."""
    pc, g, _ = make(33, Hq, Hkv, D, 128, formats, [128] * (2 * B))
    for b in range(B):
        if formats != "8bit":   # (slot b of each pair is a bf16 one in a mixed store too)
            k, v = pc.percache_kv_get(0, b)
            v[:, 40, [3, 9]] = float("inf")
            pc.percache_kv_put(0, b, k, v)
    kv = stored(pc)
    q, k, v = bf16(g.standard_normal((B, Hq, T, D))), bf16(g.standard_normal((B, Hkv, T, D))), bf16(g.standard_normal((B, Hkv, T, D)))
    v[:, :, 0, 5] = float("inf")
    v[:, :, T // 2, 7] = -float("inf")
    v[:, :, 1, 9] = -float("inf")
    parents = [random_tree(g, T, T - 1) for _ in range(B)]
    ids, used = np.array([[b, B + b] for b in range(B)]), np.array([[128, 65 + b] for b in range(B)])
    out, lse = pc.percache_attention_draft(0, q, k, v, slot_ids=ids, used_len=used, parents=parents, n_splits=n_splits, lse_out=True)
    torch.cuda.synchronize()
    assert torch.isfinite(lse[:, :, :T - 1]).all()
    got = host(out).astype(np.float64).reshape(B, T, Hq, D)
    for b in range(B):
        kc, vc = cached(kv, ids[b], used[b])
        with np.errstate(invalid="ignore"):
            want, _, size, _, _ = ref.attend(host(q[b]).astype(np.float64), kc, vc, host(k[b]).astype(np.float64), host(v[b]).astype(np.float64),
                                             ref.ancestors(parents[b]))
        fine = np.isfinite(want)
        assert not fine.all()
        assert np.array_equal(np.isnan(got[b]), np.isnan(want)) and np.array_equal(got[b][np.isinf(want)], want[np.isinf(want)])
        assert (np.abs(got[b][fine] - want[fine]) <= (2.0 ** -7 + 2.0 ** -13) * size[fine]).all()
    pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("D", [64, 128])
def test_paths_longer_than_a_launch_takes(D, formats):
    """Paths of a thousand nodes and more, which go in pieces, among short ones, with the nodes' weights; starts inside and at the ends of blocks."""
    cuts = [(0, 1500), (37, 829), (640, 1408), (5, 3), (100, 1000), (2048, 0)]
    B, T, Hkv, C = len(cuts), 1600, 2, 2048
    pc, g, kv = make(34, 2, Hkv, D, C, formats, [max(a, 1) + 3 if a < C else C for a, _ in cuts])
    k, v = bf16(g.standard_normal((B, Hkv, T, D))), bf16(3 * g.standard_normal((B, Hkv, T, D)))
    path = np.array([g.integers(0, T, T) for _ in range(B)])
    w, dw = torch.rand((B, Hkv, C), device=DEV), torch.rand((B, Hkv, T), device=DEV)
    want_w = w.clone()
    order = [4, 0, 5, 2, 1, 3]   # slot of each query
    pc.percache_kv_append_path(0, k, v, order, path, n_path=[cuts[s][1] for s in order], start=[cuts[s][0] for s in order], weights=w, draft_weights=dw)
    torch.cuda.synchronize()
    n8 = {"bf16": 0, "8bit": B, "mixed": B // 2}[formats]
    for b, s in enumerate(order):
        a, n = cuts[s]
        assert pc.percache_kv_len(0, s) == a + n
        at = torch.as_tensor(path[b, :n].astype(np.int64), device=DEV)
        want_w[s, :, a:a + n] = dw[b][:, at]
        got = pc.percache_kv_get(0, s)
        for x, new, got_x in ((0, k, got[0]), (1, v, got[1])):
            full = np.concatenate([kv[s][x][:, :a], host(new[b][:, at]).astype(np.float64)], 1)
            lo = a // 64 * 64
            if s >= B - n8 and full.shape[1] > lo:
                full[:, lo:] = kv_fp8.round_trip(full[:, lo:])
            assert np.array_equal(host(got_x), full.astype(np.float32)), (s, x)
    assert torch.equal(w, want_w)
    pc.close()


def test_weights_of_slots_none_of_whose_rows_counts():
    """A query with chunks and an empty path beside one with a long path and no chunk, without draft keys: the sums stay as they are."""
    pc, g, kv = make(35, 2, 1, 64, 192, "mixed", [190, 0])
    T = 200
    q, lse = bf16(g.standard_normal((2, 2, T, 64))), torch.zeros((2, 2, T), device=DEV)
    start = torch.rand((2, 1, 192), device=DEV)
    w = torch.full_like(start, -1.0)
    pc.percache_attention_weights(0, q, None, lse, start, w, slot_ids=[[0], [0]], used_len=[[150], [0]], n_chunks=[1, 0], path=[list(range(T))] * 2, n_path=[0, T])
    torch.cuda.synchronize()
    assert torch.equal(w[0, :, :150], start[0, :, :150]) and (w[0, :, 150:] == -1).all() and (w[1] == -1).all()
    pc.close()


class WorkspacesOf:
    """The library with a look at the workspace and the stream that a call is given."""

    def __init__(self, lib):
        self.lib, self.seen = lib, []

    def __getattr__(self, name):
        call = getattr(self.lib, name)
        if name not in ("percache_qkv_rope_draft", "percache_attention_draft", "percache_attention_weights", "percache_kv_keep"):
            return call

        def looked_at(*args):
            self.seen.append((args[-3], args[-3] + args[-2], args[-1]))
            return call(*args)
        return looked_at


def test_a_workspace_is_used_on_one_stream_only():
    """Work that is still running on one stream keeps its lists and partials whatever another one asks for, and what is given back, its memory."""
    pc, g, kv = make(36, 4, 2, 64, 128, "bf16", [128, 128, 100])
    pc.lib = WorkspacesOf(pc.lib)
    x, wqkv = bf16(g.standard_normal((1, 9, 256))), bf16(0.05 * g.standard_normal((8 * 64, 256)))
    w = torch.zeros((3, 2, 128), device=DEV)
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream()]
    results = []
    torch.cuda.synchronize()
    for n in (1, 4):   # (the second time larger ones)
        for s in streams:
            with torch.cuda.stream(s):
                q, k, v = pc.percache_qkv_rope_draft(x.expand(n, 9, 256).contiguous(), wqkv, [256] * n)
                out, lse = pc.percache_attention_draft(0, q, k, v, slot_ids=[[0, 1]] * n, lse_out=True)
                paid = pc.percache_attention_weights(0, q, k, lse, None, w, slot_ids=[[0, 1]] * n)
                pc.percache_kv_keep(0, [2], 100, w)
            torch.cuda.synchronize()
            results.append((out[0], lse[0], paid[0]))
    assert all(torch.equal(a, b) for i in (1, 2, 4, 5) for a, b in zip(results[i // 3 * 3], results[i]))
    seen = pc.lib.seen
    assert len(seen) == 24 and len({s for _, _, s in seen}) == 3
    for lo, hi, s in seen:
        assert all(s == s2 or hi <= lo2 or hi2 <= lo for lo2, hi2, s2 in seen)
    pc.close()
