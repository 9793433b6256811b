"""Drafted tokens over the cache through the C ABI -- attention of trees, projection at the nodes' positions, attention weights, accepted paths --
against the float64 reference (oracle/draft_ref.py, oracle.qkv_rope).

Bounds, from the arithmetic.  Attention: q, k, v are the same bf16 numbers on both sides; a probability is rounded to bf16 once (eight
significant bits: 2^-8 of itself), the output once (2^-8), everything else is fp32, so |error| <= (2^-7 + 2^-13) sum_j p_j |v_j| element by element.  Log-sum-exp: a score is an fp32
sum of D exact products, off by at most D 2^-24 S with S the largest sum of |q_d k_d| / sqrt(D); the exponentials (2^-22 each, with the sums of n
of them, n 2^-24) come on top, and the result, up to |lse|, is rounded a few times: (D S + n + 8 |lse| + 64) 2^-24.  A weight moves by the
error of its score and its log-sum-exp, relative: (D S + n + 16 |lse| + 128) 2^-24, and its sum over r rows by r 2^-24 more.  Copies are exact."""
import numpy as np
import pytest
import torch

import oracle
from oracle import draft_ref as ref
from oracle import kv_fp8
from paper_2601_11553_amd import workloads as wl
from paper_2601_11553_amd.binding import Percache, PercacheError

from gpu_util import DEV, bf16, check_close, host

pytestmark = pytest.mark.gpu


def make(seed, Hq, Hkv, D, C, formats, lengths, n_layers=1, max_pos=2048, hidden=256):
    """A context with one slot per length, and what its slots read back as (float64 [slots][Hkv, length, D])."""
    g = np.random.default_rng(seed)
    n = len(lengths)
    n8 = {"bf16": 0, "8bit": n, "mixed": n // 2}[formats]
    pc = Percache(n_layers=n_layers, hidden=hidden, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_slots=n, slot_capacity=C, max_pos=max_pos, n_slots_8bit=n8, device=DEV)
    for s, m in enumerate(lengths):
        if m:
            pc.percache_kv_put(n_layers - 1, s, bf16(g.standard_normal((Hkv, m, D))), bf16(g.standard_normal((Hkv, m, D))))
    return pc, g, stored(pc, n_layers - 1)


def stored(pc, layer=0):
    kv = []
    for s in range(pc.cfg.n_slots):
        if pc.percache_kv_len(layer, s):
            k, v = pc.percache_kv_get(layer, s)
            kv.append((host(k).astype(np.float64), host(v).astype(np.float64)))
        else:
            kv.append((np.zeros((pc.cfg.n_kv_heads, 0, pc.cfg.head_dim)),) * 2)
    return kv


def random_tree(g, T, live=None, reach=6):
    return [int(g.integers(max(-1, i - reach), i)) if i < (T if live is None else live) else -2 for i in range(T)]


def cached(kv, ids, used):
    return tuple(np.concatenate([kv[s][x][:, :u] for s, u in zip(ids, used)] + [kv[0][x][:, :0]], 1) for x in (0, 1))


def check_attention(pc, kv, q, k, v, ids, used, parents, layer=0, clean=None, only=None, **kw):
    """Runs the call and checks it row by row; returns lse and the reference's probabilities per query.  clean: q, k, v without the rubbish that
    the rows `only` (per query) do not look at."""
    B, Hq, T, D = q.shape
    out, lse = pc.percache_attention_draft(layer, q, k, v, slot_ids=ids, used_len=used, parents=parents, lse_out=True, **kw)
    torch.cuda.synchronize()
    o, ls = host(out).astype(np.float64).reshape(B, T, Hq, D), lse.double().cpu().numpy()
    qh, kh, vh = (host(x).astype(np.float64) for x in clean or (q, k, v))
    found = []
    for b in range(B):
        seen = ref.ancestors(parents[b] if parents is not None else [i - 1 for i in range(T)])
        kc, vc = cached(kv, ids[b] if ids is not None else [], used[b] if used is not None else [])
        want, wl_, size, S, probs = ref.attend(qh[b], kc, vc, kh[b], vh[b], seen)
        n = kc.shape[1] + T
        rows = only[b] if only else list(range(T))
        assert np.isfinite(o[b][rows]).all()
        err = (np.abs(o[b] - want) - (2.0 ** -7 + 2.0 ** -13) * size)[rows]
        print(f"query {b}: worst {err.max():.2e}", flush=True)
        assert err.max() <= 0, (b, err.max())
        wl_, ls_ = wl_[:, rows], ls[b][:, rows]
        live = np.isfinite(wl_)
        assert np.array_equal(np.isfinite(ls_), live) and (ls_[~live] == -np.inf).all()
        tol = (D * S + n + 8 * np.abs(wl_[live]) + 64) * 2.0 ** -24
        assert (np.abs(ls_[live] - wl_[live]) <= tol).all(), np.abs(ls_[live] - wl_[live]).max()
        found.append((wl_, S, n, probs))
    return lse, found


# heads, kv heads, head size, batch, nodes, used lengths of each query's chunks, capacity: rows per kv head from one to 4 x 256, lengths that end inside a
# 64-key tile, chunks of no use, queries without a cache, one token, more than 64 chunks
SHAPES = [
    (2, 2, 64, 1, 1, [[1]], 64), (2, 1, 128, 1, 1, [[]], 64), (4, 2, 64, 2, 5, [[64, 63], [1, 0]], 64), (16, 8, 128, 1, 16, [[130, 77, 128, 1]], 192),
    (6, 2, 128, 3, 11, [[65], [0], [128]], 128), (4, 2, 128, 2, 17, [[100, 64], [3, 190]], 192), (14, 2, 64, 2, 9, [[70, 0, 5], [64, 128, 128]], 128),
    (6, 2, 128, 1, 64, [[300, 511]], 512), (8, 2, 128, 2, 33, [[64, 64, 64], [1, 1, 1]], 64), (8, 1, 64, 1, 65, [[200]], 256), (4, 4, 128, 2, 130, [[129], [64]], 192),
    (4, 1, 128, 1, 256, [[90]], 128), (2, 1, 64, 1, 256, [[]], 64), (2, 1, 128, 1, 40, [[7] * 70], 64), (32, 8, 128, 8, 33, [[64, 40]] * 8, 64),
    (28, 4, 128, 1, 64, [[64] * 30], 64),
]


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}over{s[1]}x{s[2]}_b{s[3]}_t{s[4]}")
def test_attention_of_trees(shape, formats):
    Hq, Hkv, D, B, T, used, C = shape
    n_c = len(used[0])
    pc, g, kv = make(5, Hq, Hkv, D, C, formats, [C if x % 3 else max(1, C - 7) for x in range(max(2, B * n_c))], max_pos=8192)
    ids = np.arange(B * n_c).reshape(B, n_c) if n_c else np.zeros((B, 0), np.int32)
    lens = np.array([[len(kv[s][0][0]) for s in row] for row in ids]).reshape(B, n_c)
    used = np.minimum(np.array(used, np.int32).reshape(B, n_c), lens) if n_c else None
    q, k, v = bf16(1.5 * g.standard_normal((B, Hq, T, D))), bf16(g.standard_normal((B, Hkv, T, D))), bf16(g.standard_normal((B, Hkv, T, D)))
    parents = [random_tree(g, T, T - b % 3 if T > 3 else None) for b in range(B)]
    check_attention(pc, kv, q, k, v, ids if n_c else None, used, parents)
    pc.close()


@pytest.mark.parametrize("T", [1, 2, 16, 31, 64, 100])
def test_a_sequence_without_parents_is_causal(T):
    pc, g, kv = make(6, 4, 2, 128, 128, "bf16", [128, 90])
    q, k, v = bf16(g.standard_normal((1, 4, T, 128))), bf16(g.standard_normal((1, 2, T, 128))), bf16(g.standard_normal((1, 2, T, 128)))
    check_attention(pc, kv, q, k, v, [[0, 1]], [[128, 90]], None)
    chain = pc.percache_attention_draft(0, q, k, v, slot_ids=[[0, 1]], parents=[[i - 1 for i in range(T)]])[0]
    plain = pc.percache_attention_reuse(0, q, k, v, [[0, 1]])
    torch.cuda.synchronize()
    check_close(host(chain), host(plain), f"T={T}")
    pc.close()


@pytest.mark.parametrize("Hq,Hkv,T", [(4, 2, 6), (8, 2, 48)])
def test_partitions_give_the_same(Hq, Hkv, T):
    pc, g, kv = make(7, Hq, Hkv, 128, 256, "mixed", [256] * 4)
    q, k, v = bf16(g.standard_normal((1, Hq, T, 128))), bf16(g.standard_normal((1, Hkv, T, 128))), bf16(g.standard_normal((1, Hkv, T, 128)))
    parents = [random_tree(g, T, T - 1)]
    for n in (1, 2, 3, 5, 8):
        check_attention(pc, kv, q, k, v, [[0, 1, 2, 3]], [[256, 255, 1, 256]], parents, n_splits=n)
    pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("Hq,Hkv,D,T,B", [(4, 2, 64, 5, 1), (4, 2, 128, 7, 1), (8, 2, 64, 20, 2), (6, 2, 128, 20, 2), (32, 8, 128, 33, 8), (2, 2, 128, 40, 1), (8, 8, 64, 140, 8)])
def test_what_a_row_does_not_see_takes_no_part(Hq, Hkv, D, T, B, formats):
    """Infinities and NaN behind the used lengths, in other branches and in padding; scores of the type's lowest values."""
    pc, g, _ = make(8, Hq, Hkv, D, 128, formats, [128] * (2 * B))
    kv = stored(pc)
    for s in range(2 * B):                      # the slots again, with rubbish behind token 70
        k, v = (bf16(x) for x in kv[s])
        for x in (k, v):
            x[:, 70:90] = float("nan")
            x[:, 90:110] = float("inf")
            x[:, 110:] = -float("inf")
        if formats == "bf16" or s < B and formats == "mixed":
            pc.percache_kv_put(0, s, k, v)
    q, k, v = bf16(g.standard_normal((B, Hq, T, D))), bf16(g.standard_normal((B, Hkv, T, D))), bf16(g.standard_normal((B, Hkv, T, D)))
    parents = [random_tree(g, T, T - 2, reach=3) for _ in range(B)]
    for b in range(B):
        seen = ref.ancestors(parents[b])
        bad = [i for i in range(T - 2) if not any(i in seen[j] for j in range(T) if j != i)]   # leaves: nobody else looks at them
        for n, i in enumerate(bad[:len(bad) // 2] + [T - 2, T - 1]):
            k[b, :, i], v[b, :, i] = [(float("nan"), float("inf")), (3e38, float("nan")), (float("-inf"), -3e38)][n % 3]
            if i >= T - 2:
                q[b, :, i] = float("nan")
    ids, used = np.arange(2 * B).reshape(B, 2), np.array([[70, 64 + b % 6] for b in range(B)])
    clean = [x.clone() for x in (q, k, v)]
    for x in clean:
        x[~torch.isfinite(x)] = 0.0
        x[x.abs() > 1e30] = 0.0
    fine = [[i for i in range(T - 2) if all(torch.equal(x[b, :, i], y[b, :, i]) for x, y in zip((k, v), clean[1:]))] for b in range(B)]
    assert all(len(rows) > T // 3 for rows in fine)
    check_attention(pc, kv, q, k, v, ids, used, parents, clean=clean, only=[rows + [T - 2, T - 1] for rows in fine])
    out, lse = pc.percache_attention_draft(0, q, k, v, slot_ids=ids, used_len=used, parents=parents, lse_out=True)
    torch.cuda.synchronize()
    assert (out[:, T - 2:] == 0).all() and (lse[:, :, T - 2:] == -float("inf")).all()
    # their weights likewise
    w = torch.zeros((2 * B, Hkv, 128), device=DEV)
    rows = fine
    n_path = [len(r) for r in rows]
    path = np.array([r + [0] * (T - len(r)) for r in rows])
    d = pc.percache_attention_weights(0, q, k, lse, None, w, slot_ids=ids, used_len=used, parents=parents, path=path, n_path=n_path)
    torch.cuda.synchronize()
    for b in range(B):
        for c in range(2):
            assert torch.isfinite(w[2 * b + c, :, :used[b, c]]).all() and (w[2 * b + c, :, used[b, c]:] == 0).all()
        unseen = [j for j in range(T) if not any(j in ref.ancestors(parents[b])[i] for i in rows[b])]
        assert torch.isfinite(d[b]).all() and (d[b][:, unseen] == 0).all()
    pc.close()


def test_batches_of_nothing_but_padding():
    pc, g, kv = make(9, 4, 2, 64, 64, "bf16", [64, 64])
    for T in (3, 40):
        q, k, v = bf16(g.standard_normal((2, 4, T, 64))), bf16(g.standard_normal((2, 2, T, 64))), bf16(g.standard_normal((2, 2, T, 64)))
        q[:], k[:], v[:] = float("nan"), float("inf"), float("nan")
        out, lse = pc.percache_attention_draft(0, q, k, v, slot_ids=[[0], [1]], parents=[[-2] * T] * 2, lse_out=True)
        w = torch.full((2, 2, 64), 0.5, device=DEV)
        d = pc.percache_attention_weights(0, q, k, lse, w, w, slot_ids=[[0], [1]], parents=[[-2] * T] * 2)
        torch.cuda.synchronize()
        assert (out == 0).all() and (lse == -float("inf")).all() and (w == 0.5).all() and (d == 0).all()
    pc.close()


@pytest.mark.parametrize("H,Hq,Hkv,D,B,T,seq", [(256, 4, 2, 64, 1, 1, False), (256, 4, 2, 64, 3, 13, False), (512, 4, 2, 128, 2, 40, False), (1024, 16, 8, 128, 1, 16, False),
                                               (256, 4, 2, 128, 2, 150, False), (512, 8, 2, 128, 8, 200, True), (320, 2, 1, 128, 1, 7, True)])
def test_projection_at_the_positions_of_the_nodes(H, Hq, Hkv, D, B, T, seq):
    pc = Percache(n_layers=1, hidden=H, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_slots=1, slot_capacity=64, max_pos=900, device=DEV)
    g = np.random.default_rng(10 + T)
    x, w = bf16(g.standard_normal((B, T, H))), bf16(0.02 * g.standard_normal(((Hq + 2 * Hkv) * D, H)))
    parents = None if seq else [random_tree(g, T, max(1, T - b)) for b in range(B)]
    pos0 = [int(g.integers(0, 900 - T + 1)) for _ in range(B)]
    if not seq:
        pos0[0] = 899 - max(ref.depths(parents[0]))   # (the deepest node at the last position)
    q, k, v = pc.percache_qkv_rope_draft(x, w, pos0, parents=parents)
    torch.cuda.synchronize()
    for b in range(B):
        depth = list(range(T)) if seq else ref.depths(parents[b])
        for i in range(T):
            if T > 20 and i % 7:
                continue
            qr, kr, vr = oracle.qkv_rope(host(x[b, i:i + 1]), host(w), Hq, Hkv, D, pos0[b] + depth[i], 10000.0)
            for got, want in ((q[b, :, i], qr), (k[b, :, i], kr), (v[b, :, i], vr)):
                want = np.asarray(want).reshape(got.shape)
                # one bf16 rounding of an fp32 sum; a rotation by a table entry rounded to fp32
                assert (np.abs(host(got) - want) <= 2.0 ** -8 * np.abs(want) + 1e-4).all()
    pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("Hq,Hkv,D,B,T,n_c,paths", [(4, 2, 64, 1, 1, 1, False), (4, 2, 128, 3, 9, 2, True), (16, 8, 128, 2, 20, 3, True), (14, 2, 64, 2, 33, 4, False),
                                                     (6, 2, 128, 4, 70, 2, False), (6, 2, 128, 2, 256, 2, True), (2, 1, 64, 1, 5, 66, True)])
def test_weights(Hq, Hkv, D, B, T, n_c, paths, formats):
    """Chunk 0 shared by every query (with different used lengths), the others their own, one named twice by a query."""
    n = 1 + B * (n_c - 1)
    C = 128
    pc, g, kv = make(11, Hq, Hkv, D, C, formats, [C - s % 5 for s in range(max(n, 2))], max_pos=16384)
    ids = np.array([[0] + [1 + b * (n_c - 1) + c for c in range(n_c - 1)] for b in range(B)])
    used = np.array([[len(kv[s][0][0]) - (3 * b if c == 0 else c % 3 * 30) for c, s in enumerate(ids[b])] for b in range(B)])
    if n_c > 2:
        ids[0, 2], used[0, 2] = ids[0, 1], 17
        used[-1, 1] = 0
    q, k, v = bf16(2 * g.standard_normal((B, Hq, T, D))), bf16(g.standard_normal((B, Hkv, T, D))), bf16(g.standard_normal((B, Hkv, T, D)))
    parents = [random_tree(g, T, T if b % 2 else max(1, T - 2)) for b in range(B)]
    lse, found = check_attention(pc, kv, q, k, v, ids, used, parents)
    if paths:
        n_path = [0 if b == 1 and B > 2 else min(T, 1 + b + 3) for b in range(B)]
        path = np.array([g.permutation(T)[:min(T, B + 4)].tolist() + [0] * (B + 4) for _ in range(B)])[:, :min(T, B + 4)]
        rows = [path[b, :n_path[b]].tolist() for b in range(B)]
        kw = dict(path=path, n_path=n_path)
    else:
        rows, kw = [list(range(T))] * B, {}
    start = torch.rand((max(n, 2), Hkv, C), device=DEV)
    out = start.clone()
    draft = pc.percache_attention_weights(0, q, k, lse, start, out, slot_ids=ids, used_len=used, parents=parents, **kw)
    torch.cuda.synchronize()
    want, paid = start.double().cpu().numpy(), np.zeros((max(n, 2), Hkv, C))
    rel = 0.0
    for b in range(B):
        wl_, S, keys, probs = found[b]
        c, d = ref.weights(probs, Hq, Hkv, T, keys - T, rows[b])
        lo = 0
        for s, u in zip(ids[b], used[b]):
            paid[s, :, :u] += c[:, lo:lo + u]
            lo += u
        live = np.isfinite(wl_)
        r = (D * S + keys + 16 * np.abs(wl_[live]).max(initial=0) + 128 + B * Hq // Hkv * max(1, len(rows[b]))) * 2.0 ** -24
        rel = max(rel, r)
        got = draft[b].double().cpu().numpy()
        assert (np.abs(got - d) <= r * d).all(), (np.abs(got - d) / np.maximum(d, 1e-300)).max()
    got = out.double().cpu().numpy()
    assert (np.abs(got - want - paid) <= rel * paid + 2.0 ** -23 * (want + paid)).all()
    assert np.array_equal(got[paid == 0], want[paid == 0])
    # in place, from zero, and without the draft keys: the same sums, bit for bit
    again = start.clone()
    d2 = pc.percache_attention_weights(0, q, k, lse, again, again, slot_ids=ids, used_len=used, parents=parents, **kw)
    zero = torch.zeros_like(start)
    none = pc.percache_attention_weights(0, q, None, lse, None, zero, slot_ids=ids, used_len=used, parents=parents, **kw)
    ref0 = torch.zeros_like(start)
    pc.percache_attention_weights(0, q, k, lse, ref0, ref0, slot_ids=ids, used_len=used, parents=parents, **kw)
    torch.cuda.synchronize()
    assert torch.equal(again, out) and torch.equal(d2, draft) and none is None and torch.equal(zero, ref0)
    pc.close()


def test_weights_of_a_sequence_longer_than_a_tree_may_be():
    """Rows of a prompt: 300 of them, no parents; lse from the reference."""
    Hq, Hkv, D, T = 4, 2, 64, 300
    pc, g, kv = make(12, Hq, Hkv, D, 128, "bf16", [100, 128])
    q, k, v = bf16(g.standard_normal((1, Hq, T, D))), bf16(g.standard_normal((1, Hkv, T, D))), bf16(g.standard_normal((1, Hkv, T, D)))
    lse, found = check_attention(pc, kv, q, k, v, [[0, 1]], [[100, 128]], None)
    w = torch.zeros((2, Hkv, 128), device=DEV)
    d = pc.percache_attention_weights(0, q, k, lse, None, w, slot_ids=[[0, 1]])
    torch.cuda.synchronize()
    c, dd = ref.weights(found[0][3], Hq, Hkv, T, 228, range(T))
    r = (D * found[0][1] + 228 + T + 16 * np.abs(found[0][0]).max() + 128 + 2 * T) * 2.0 ** -24
    assert (np.abs(torch.cat([w[0, :, :100], w[1]], 1).double().cpu().numpy() - c) <= r * c).all()
    assert (np.abs(d[0].double().cpu().numpy() - dd) <= r * dd).all()
    pc.close()


@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("D,T,B,cuts", [(64, 5, 2, [(0, 1), (63, 2)]), (128, 16, 4, [(60, 9), (64, 0), (100, 4), (127, 1)]), (128, 80, 3, [(10, 70), (37, 0), (0, 0)]),
                                        (64, 200, 2, [(1, 127), (128, 0)]), (128, 12, 40, [(b, 12) for b in range(40)])])
def test_accepted_paths(D, T, B, cuts, formats):
    Hkv, C = 2, 128
    pc, g, kv = make(13, 2, Hkv, D, C, formats, [128] * B)
    k, v = bf16(g.standard_normal((B, Hkv, T, D))), bf16(3 * g.standard_normal((B, Hkv, T, D)))
    most = max(1, max(n for _, n in cuts))
    n_path, start = [n for _, n in cuts], [a for a, _ in cuts]
    path = np.array([g.integers(0, T, most) for _ in range(B)])
    w, dw = torch.rand((B, Hkv, C), device=DEV), torch.rand((B, Hkv, T), device=DEV)
    want_w = w.clone()
    slots = list(range(B))
    pc.percache_kv_append_path(0, k, v, slots, path, n_path=n_path, start=start, weights=w, draft_weights=dw)
    torch.cuda.synchronize()
    n8 = {"bf16": 0, "8bit": B, "mixed": B // 2}[formats]
    for b, (a, n) in enumerate(cuts):
        assert pc.percache_kv_len(0, b) == a + n
        at = torch.as_tensor(path[b, :n].astype(np.int64), device=DEV)
        want_w[b, :, a:a + n] = dw[b][:, at]
        if a + n == 0:
            continue
        got = pc.percache_kv_get(0, b)
        for x, new, got_x in ((0, k, got[0]), (1, v, got[1])):
            full = np.concatenate([kv[b][x][:, :a], host(new[b][:, at]).astype(np.float64)], 1)
            if b >= B - n8:
                lo = a // 64 * 64
                full[:, lo:] = kv_fp8.round_trip(full[:, lo:]) if full.shape[1] > lo else full[:, lo:]
            assert np.array_equal(host(got_x), full.astype(np.float32)), (b, x)
    assert torch.equal(w, want_w)
    # attention over the slots reads the same as over slots written whole (the padding behind the last token stays finite)
    live = [b for b in range(B) if cuts[b][0] + cuts[b][1]]
    q = bf16(g.standard_normal((len(live), 2, 5, D)))
    kf, vf = bf16(g.standard_normal((len(live), Hkv, 5, D))), bf16(g.standard_normal((len(live), Hkv, 5, D)))
    a0 = pc.percache_attention_reuse(0, q, kf, vf, [[b] for b in live])
    whole = Percache(n_layers=1, hidden=256, n_q_heads=2, n_kv_heads=Hkv, head_dim=D, n_slots=B, slot_capacity=C, max_pos=2048, n_slots_8bit=n8, device=DEV)
    for b in live:
        whole.percache_kv_put(0, b, *pc.percache_kv_get(0, b))
    a1 = whole.percache_attention_reuse(0, q, kf, vf, [[b] for b in live])
    torch.cuda.synchronize()
    assert torch.equal(a0, a1)
    pc.close()
    whole.close()


def test_paths_behind_the_last_token_and_skipped_slots():
    pc, g, kv = make(14, 2, 2, 64, 64, "bf16", [10, 0, 63])
    k, v = bf16(g.standard_normal((3, 2, 4, 64))), bf16(g.standard_normal((3, 2, 4, 64)))
    pc.percache_kv_append_path(0, k, v, [2, -1, 0], [[1, 0], [3, 3], [0, 3]], n_path=[1, 2, 2])
    torch.cuda.synchronize()
    assert [pc.percache_kv_len(0, s) for s in range(3)] == [12, 0, 64]
    assert torch.equal(pc.percache_kv_get(0, 2)[0][:, 63], k[0, :, 1]) and torch.equal(pc.percache_kv_get(0, 0)[1][:, 10:], v[2][:, [0, 3]])
    pc.close()


def test_calls_on_a_stream_of_their_own():
    pc, g, kv = make(15, 4, 2, 128, 128, "bf16", [128, 128])
    q, k, v = bf16(g.standard_normal((1, 4, 40, 128))), bf16(g.standard_normal((1, 2, 40, 128))), bf16(g.standard_normal((1, 2, 40, 128)))
    parents = [random_tree(g, 40)]
    want = pc.percache_attention_draft(0, q, k, v, slot_ids=[[0, 1]], parents=parents, lse_out=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = pc.percache_attention_draft(0, q, k, v, slot_ids=[[0, 1]], parents=parents, lse_out=True)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    pc.close()


def test_stores_of_more_than_2_to_the_31_elements():
    """The last slots of a store of 2^31 + elements each for K and V."""
    Hq, Hkv, D, C = 4, 2, 128, 1024
    n = (1 << 31) // (Hkv * C * D) + 4
    pc = Percache(n_layers=1, hidden=256, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_slots=n, slot_capacity=C, max_pos=4096, device=DEV)
    g = np.random.default_rng(16)
    a, b = n - 2, n - 1
    for s, m in ((a, 200), (b, 130)):
        pc.percache_kv_put(0, s, bf16(g.standard_normal((Hkv, m, D))), bf16(g.standard_normal((Hkv, m, D))))
    kv = {s: tuple(host(x).astype(np.float64) for x in pc.percache_kv_get(0, s)) for s in (a, b)}
    kv[0] = kv[a]
    for T in (4, 40):
        q, k, v = bf16(g.standard_normal((1, Hq, T, D))), bf16(g.standard_normal((1, Hkv, T, D))), bf16(g.standard_normal((1, Hkv, T, D)))
        parents = [random_tree(g, T)]
        lse, found = check_attention(pc, kv, q, k, v, [[a, b]], [[200, 130]], parents)
        w = torch.zeros((n, Hkv, C), device=DEV)
        pc.percache_attention_weights(0, q, k, lse, w, w, slot_ids=[[a, b]], parents=parents)
        torch.cuda.synchronize()
        c, _ = ref.weights(found[0][3], Hq, Hkv, T, 330, range(T))
        assert np.allclose(torch.cat([w[a, :, :200], w[b, :, :130]], 1).cpu().numpy(), c, rtol=1e-4)
        assert float(w[:a].abs().max()) == 0
    pc.percache_kv_append_path(0, k, v, [b], [[2, 3]], start=[129])
    idx = pc.percache_kv_keep(0, [a], 50, w, n_first=2, n_last=3)
    torch.cuda.synchronize()
    assert torch.equal(pc.percache_kv_get(0, b)[0][:, 129:], k[0][:, [2, 3]])
    got = host(pc.percache_kv_get(0, a)[0])
    for h in range(Hkv):
        assert np.array_equal(got[h], kv[a][0][h][idx[0, h].cpu().numpy()].astype(np.float32))
    pc.close()


def test_refusals_have_no_effect():
    pc, g, kv = make(17, 4, 2, 64, 128, "bf16", [128, 100, 0], max_pos=300)
    T = 6
    q, k, v = bf16(g.standard_normal((2, 4, T, 64))), bf16(g.standard_normal((2, 2, T, 64))), bf16(g.standard_normal((2, 2, T, 64)))
    x, w = bf16(g.standard_normal((2, T, 256))), bf16(g.standard_normal((8 * 64, 256)))
    tree = [[-1, 0, 1, 0, -2, -2]] * 2
    lse = torch.zeros((2, 4, T), device=DEV)
    acc = torch.full((3, 2, 128), 0.25, device=DEV)
    dw = torch.zeros((2, 2, T), device=DEV)
    att = lambda **kw: pc.percache_attention_draft(0, q, k, v, **{**dict(slot_ids=[[0], [1]], parents=tree), **kw})   # noqa: E731
    wgt = lambda **kw: pc.percache_attention_weights(0, q, k, lse, acc, acc, **{**dict(slot_ids=[[0], [1]], parents=tree), **kw})   # noqa: E731
    app = lambda **kw: pc.percache_kv_append_path(0, k, v, **{**dict(append_slots=[1, -1], path=[[0, 1]] * 2), **kw})   # noqa: E731
    keep = lambda **kw: pc.percache_kv_keep(0, **{**dict(slots=[0], keep=10, weights=acc), **kw})   # noqa: E731
    cases = [
        (lambda: att(parents=[[0, -1, 0, 0, 0, 0]] * 2), -1), (lambda: att(parents=[[-3] + [-1] * 5] * 2), -1), (lambda: att(parents=[[-2, 0, -1, -1, -1, -1]] * 2), -1),
        (lambda: att(slot_ids=[[0], [2]]), -3), (lambda: att(slot_ids=[[0], [3]]), -3), (lambda: att(used_len=[[1], [101]]), -4), (lambda: att(n_splits=1000), -1),
        (lambda: pc.percache_attention_draft(1, q, k, v), -3),
        (lambda: pc.percache_attention_draft(0, *(torch.zeros((1, h, 257, 64), dtype=torch.bfloat16, device=DEV) for h in (4, 2, 2)), parents=[[-1] * 257]), -2),
        (lambda: pc.percache_qkv_rope_draft(x, w, [0, 295], parents=[[-1, 0, 1, 2, 3, 4]] * 2), -4), (lambda: pc.percache_qkv_rope_draft(x, w, [-1, 0], parents=tree), -4),
        (lambda: pc.percache_qkv_rope_draft(x, w, [295, 0]), -4), (lambda: pc.percache_qkv_rope_draft(x, w, [0, 0], parents=[[5] * T] * 2), -1),
        (lambda: wgt(path=[[0, 6]] * 2), -1), (lambda: wgt(path=[[0, 1]] * 2, n_path=[3, 0]), -1), (lambda: wgt(path=[[0] * 7] * 2), -1), (lambda: wgt(slot_ids=[[2], [0]]), -3),
        (lambda: app(path=[[0, -1]] * 2), -1), (lambda: app(append_slots=[1, 1]), -1), (lambda: app(append_slots=[3, -1]), -3), (lambda: app(start=[101, 0]), -4),
        (lambda: app(append_slots=[0, -1]), -4), (lambda: app(draft_weights=dw), -1), (lambda: app(n_path=[-1, 0]), -1),
        (lambda: keep(keep=0), -4), (lambda: keep(keep=129), -4), (lambda: keep(n_first=6, n_last=5), -1), (lambda: keep(n_first=-1), -1), (lambda: keep(slots=[2]), -3),
        (lambda: keep(slots=[0, 0]), -1), (lambda: keep(slots=[0, 1], dst_slots=[1, 2]), -1), (lambda: keep(dst_slots=[3]), -3),
    ]
    for n, (call, status) in enumerate(cases):
        with pytest.raises(PercacheError) as e:
            call()
        assert e.value.status == status, (n, str(e.value))
    shapes = [lambda: pc.percache_attention_draft(0, q.transpose(2, 3).contiguous().transpose(2, 3), k, v), lambda: pc.percache_attention_draft(0, q.float(), k, v),
              lambda: pc.percache_attention_weights(0, q, k, lse.double(), acc, acc), lambda: keep(weights=acc[:2]), lambda: pc.percache_kv_append_path(0, k, v[:, :1], [0, 1], [[0]] * 2)]
    for call in shapes:
        with pytest.raises(ValueError):
            call()
    # a workspace that is too small, or out of line
    need = pc.lib.percache_draft_workspace_bytes(pc.ctx, 2, T, 0)
    ws = torch.zeros(need + 256, dtype=torch.uint8, device=DEV)
    at = (ws.data_ptr() + 255) // 256 * 256
    for ptr, size, status in ((at, need - 1, -5), (at + 64, need, -1), (None, need, -5)):
        st = pc.lib.percache_attention_draft(pc.ctx, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), 2, T, None, None, np.zeros(2, np.int32).ctypes.data_as(
            __import__("ctypes").POINTER(__import__("ctypes").c_int32)), 0, None, 0, q.data_ptr(), None, ptr, size, None)
        assert st == status
    torch.cuda.synchronize()
    assert [pc.percache_kv_len(0, s) for s in range(3)] == [128, 100, 0] and (acc == 0.25).all()
    now = stored(pc)
    assert all(np.array_equal(a[x], b[x]) for a, b in zip(now, kv) for x in (0, 1))
    pc.close()
