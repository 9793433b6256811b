"""Attention of packed prompts through the C ABI against the float64 reference (oracle/packed_ref.py).

Bounds, from the arithmetic: q, k, v are the same bf16 numbers on both sides; a probability is rounded to bf16 once (2^-8 of itself), the output once
(2^-8), everything else is fp32, so |error| <= (2^-7 + 2^-13) sum_j p_j |v_j| element by element.  Log-sum-exp: a score is an fp32 sum of D exact
products, off by at most D 2^-24 S with S the largest sum of |q_d k_d| / sqrt(D); the exponentials and their sum of n add n 2^-24, and the result is
rounded a few times: (D S + n + 8 |lse| + 64) 2^-24."""
import numpy as np
import pytest
import torch

from oracle import packed_ref as ref

from gpu_util import DEV, bf16, host
from test_gpu_draft import cached, make, stored

pytestmark = pytest.mark.gpu


def packed(g, Hq, Hkv, D, n):
    return bf16(1.5 * g.standard_normal((Hq, n, D))), bf16(g.standard_normal((Hkv, n, D))), bf16(g.standard_normal((Hkv, n, D)))


def check(pc, kv, q, k, v, start, ids=None, used=None, clean=None, skip=(), **kw):
    """Runs the call and checks every request; rows of nobody must stay what they were.  clean: q, k, v without the rubbish that no row outside `skip`
    (packed rows) looks at."""
    Hq, N, D = q.shape
    out = torch.full((N, Hq * D), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((Hq, N), 7.0, dtype=torch.float32, device=DEV)
    pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids, used_len=used, attn_out=out, lse_out=lse, **kw)
    torch.cuda.synchronize()
    o, ls = host(out).astype(np.float64).reshape(N, Hq, D), lse.double().cpu().numpy()
    qh, kh, vh = (host(x).astype(np.float64) for x in clean or (q, k, v))
    mine = np.zeros(N, bool)
    for s in range(len(start) - 1):
        a, b = int(start[s]), int(start[s + 1])
        if a == b:
            continue
        mine[a:b] = True
        kc, vc = cached(kv, ids[s] if ids is not None else [], used[s] if used is not None else [])
        want, wl, size, S = ref.attend(qh[:, a:b], kh[:, a:b], vh[:, a:b], kc, vc)
        rows = [i for i in range(b - a) if a + i not in skip]
        got, gl = o[a:b], ls[:, a:b]
        assert np.isfinite(got[rows]).all() and np.isfinite(gl[:, rows]).all(), (s, np.argwhere(~np.isfinite(got[rows]))[:5])
        err = (np.abs(got - want) - (2.0 ** -7 + 2.0 ** -13) * size)[rows]
        assert err.max() <= 0, (s, a, b, err.max(), np.argwhere(err > 0)[:5], (err > 0).sum())
        tol = (D * S + kc.shape[1] + b - a + 8 * np.abs(wl) + 64) * 2.0 ** -24
        assert (np.abs(gl - wl) <= tol)[:, rows].all(), (s, np.abs(gl - wl)[:, rows].max())
    assert (o[~mine] == 7).all() and (ls[:, ~mine] == 7).all()
    return out, lse


# heads, kv heads, head size, lengths, used lengths of every request's chunks, capacity.  Rows per kv head on both sides of 16, 32 and 256 and their
# multiples, lengths on both sides of a tile, none, one; chunks that end inside a tile, of no use, more than 64 of them; head groups 1 to 8
SHAPES = [
    (2, 2, 64, [1], None, 64),
    (2, 1, 128, [1], [[64]], 64),
    (4, 2, 128, [0, 1, 0, 3, 0], None, 64),
    (16, 8, 128, [9, 90, 33, 64, 65], None, 64),
    (4, 2, 64, [63, 64, 65, 127, 128, 129], None, 64),
    (24, 8, 128, [1, 1, 40, 1], [[130, 0, 5], [192, 64, 1], [65, 190, 128], [0, 0, 0]], 192),
    (14, 2, 64, [37, 1, 5, 200], [[70, 0, 5], [64, 128, 128], [1, 1, 1], [127, 2, 128]], 128),
    (4, 1, 128, [8, 64, 72, 136], None, 64),
    (28, 4, 128, [150, 1, 36], [[64, 3], [63, 65], [128, 128]], 128),
    (8, 1, 64, [3, 300, 31], [[200], [255], [256]], 256),
    (3, 3, 128, [257, 15, 16, 17, 31, 32], [[129], [64], [1], [190], [0], [192]], 192),
    (2, 1, 128, [5, 200], [[7] * 70, [64, 1] * 35], 64),
    (32, 8, 128, [1] * 12, [[64, 40]] * 12, 64),
    (32, 8, 64, [700, 2, 411], None, 64),
    (6, 2, 128, [600], [[511, 300]], 512),
]
IDS = [f"{s[0]}over{s[1]}x{s[2]}_" + "_".join(map(str, s[3][:4])) + ("_cached" if s[4] else "") for s in SHAPES]


def build(shape, formats, seed=41, gap=(0, 0)):
    Hq, Hkv, D, T, used, C = shape
    B = len(T)
    n_c = len(used[0]) if used else 0
    pc, g, kv = make(seed, Hq, Hkv, D, C, formats, [C if x % 3 else max(1, C - 7) for x in range(max(2, B * n_c))], max_pos=16384)
    ids = np.random.default_rng(seed).permutation(B * n_c).reshape(B, n_c) if n_c else None
    if used:
        used = np.minimum(np.array(used, np.int32), np.array([[kv[s][0].shape[1] for s in row] for row in ids]))
    start = gap[0] + np.concatenate([[0], np.cumsum(T)])
    q, k, v = packed(g, Hq, Hkv, D, int(start[-1]) + gap[1])
    return pc, g, kv, q, k, v, start, ids, used


@pytest.mark.parametrize("shape,formats", [pytest.param(s, f, id=f"{name}-{f}") for s, name in zip(SHAPES, IDS) for f in (("bf16", "8bit", "mixed") if s[4] else ("bf16",))])
def test_requests_of_any_lengths(shape, formats):
    pc, g, kv, q, k, v, start, ids, used = build(shape, formats)
    check(pc, kv, q, k, v, start, ids, used)
    pc.close()


@pytest.mark.parametrize("n_splits", [1, 2, 3, 7])
@pytest.mark.parametrize("formats", ["bf16", "mixed"])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (1, 5, 6, 8, 10, 14)], ids=[IDS[i] for i in (1, 5, 6, 8, 10, 14)])
def test_partitions_of_the_key_axis(shape, formats, n_splits):
    pc, g, kv, q, k, v, start, ids, used = build(shape, formats, seed=42, gap=(5, 70))
    n_splits = min(n_splits, pc.lib.percache_packed_max_splits(pc.ctx, len(start) - 1, q.shape[1]))
    check(pc, kv, q, k, v, start, ids, used, n_splits=n_splits)
    pc.close()


@pytest.mark.parametrize("gap", [(0, 9), (13, 0), (1, 300)])
def test_rows_of_nobody_stay_as_they_are(gap):
    """Rows before the first and behind the last request hold NaN: nothing reads or writes them."""
    for shape in (SHAPES[3], SHAPES[4], SHAPES[5], SHAPES[10]):
        pc, g, kv, q, k, v, start, ids, used = build(shape, "bf16", gap=gap)
        for x in (q, k, v):
            x[:, :gap[0]] = float("nan")
            x[:, int(start[-1]):] = float("nan")
        check(pc, kv, q, k, v, start, ids, used)
        pc.close()


def test_what_stands_behind_used_lengths_takes_no_part():
    """Tokens of a slot behind the used length are infinite or NaN (bf16 slots)."""
    for Hq, Hkv, D, T in ((6, 2, 128, [1, 50, 200]), (4, 4, 64, [1, 20, 130])):
        pc, g, _ = make(43, Hq, Hkv, D, 192, "bf16", [192] * 6)
        for s in range(6):
            k, v = pc.percache_kv_get(0, s)
            n = 192 - 3 - 20 * s
            k[:, n:], v[:, n:] = float("nan"), float("inf")
            v[:, n + 1:, ::3] = float("nan")
            pc.percache_kv_put(0, s, k, v)
        kv = stored(pc)
        ids = np.arange(6).reshape(3, 2)
        used = np.array([[192 - 3 - 20 * s for s in row] for row in ids], np.int32)
        start = np.concatenate([[0], np.cumsum(T)])
        q, k, v = packed(g, Hq, Hkv, D, int(start[-1]))
        check(pc, kv, q, k, v, start, ids, used)
        check(pc, kv, q, k, v, start, ids, used, n_splits=2)
        pc.close()


@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 128), (6, 2, 128), (14, 2, 64), (8, 1, 64)])
@pytest.mark.parametrize("formats", ["bf16", "mixed"])
def test_rubbish_in_later_rows_takes_no_part(Hq, Hkv, D, formats):
    """Some rows' K and V are infinite or NaN: the rows of their request before them, and all other requests, are what they are without it."""
    T, C = [1, 40, 70, 300, 130], 128
    pc, g, kv = make(44, Hq, Hkv, D, C, formats, [C] * 5, max_pos=8192)
    ids, used = np.arange(5).reshape(5, 1), np.array([[1], [65], [128], [100], [0]])
    start = np.concatenate([[0], np.cumsum(T)])
    q, k, v = packed(g, Hq, Hkv, D, int(start[-1]))
    clean = tuple(x.clone() for x in (q, k, v))
    skip = set()
    for s, i, kx, vx in ((1, 39, float("nan"), float("inf")), (2, 63, 1.0, float("nan")), (3, 70, float("inf"), -float("inf")), (3, 299, 0.0, float("nan")), (4, 64, 2.0, float("inf"))):
        row = int(start[s]) + i
        k[:, row], v[:, row] = kx, vx
        v[:, row, 1::2] = 1.0
        skip |= set(range(row, int(start[s + 1])))
    for n_splits in (0, 1, 3):
        n_splits = min(n_splits, pc.lib.percache_packed_max_splits(pc.ctx, 5, q.shape[1]))
        check(pc, kv, q, k, v, start, ids, used, clean=clean, skip=skip, n_splits=n_splits)
    pc.close()


@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (14, 2, 64)])
def test_infinite_values_that_a_row_sees(Hq, Hkv, D):
    """V infinite in one dimension of one token: infinite there for every row that sees it, the usual numbers elsewhere."""
    T = [3, 150, 400]
    pc, g, kv = make(45, Hq, Hkv, D, 64, "bf16", [64, 64])
    start = np.concatenate([[0], np.cumsum(T)])
    q, k, v = packed(g, Hq, Hkv, D, int(start[-1]))
    want = pc.percache_attention_packed(0, q, k, v, start)[0]
    marks = [(0, 1, 5), (1, 70, 7), (2, 0, 9), (2, 255, 3)]
    for s, i, d in marks:
        v[:, int(start[s]) + i, d] = float("inf")
    got = pc.percache_attention_packed(0, q, k, v, start)[0]
    torch.cuda.synchronize()
    got, want = host(got).reshape(-1, Hq, D), host(want).reshape(-1, Hq, D)
    hit = np.zeros(got.shape, bool)
    for s, i, d in marks:
        hit[int(start[s]) + i:int(start[s + 1]), :, d] = True
    assert (got[hit] == np.inf).all()
    # (rows computed again, key by key, take the unrounded probabilities: both are off by at most 2^-7 of sum p |v|, here at most max |v|)
    assert np.abs(got - want)[~hit].max() <= 2.0 ** -6 * float(host(v)[np.isfinite(host(v))].max())
    pc.close()


def test_peaked_and_flat_rows():
    """Scores of +-100 (one key takes all) and rows of equal keys; the reference exponent moves in the middle of a walk."""
    Hq, Hkv, D, T = 4, 2, 128, [200, 1, 500]
    pc, g, kv = make(46, Hq, Hkv, D, 128, "bf16", [128] * 3)
    start = np.concatenate([[0], np.cumsum(T)])
    q, k, v = packed(g, Hq, Hkv, D, int(start[-1]))
    q = q * 8
    k[:, 40:60] = 0
    k[:, 300] *= 4
    check(pc, kv, q, k, v, start, np.arange(3).reshape(3, 1), np.array([[128], [70], [3]]))
    pc.close()


def test_long_prompts_agree_with_the_rectangular_call():
    """Requests of equal length through both calls (the same bound twice)."""
    Hq, Hkv, D, B, T = 8, 2, 128, 3, 1500
    pc, g, kv = make(47, Hq, Hkv, D, 512, "bf16", [512] * 6, max_pos=4096)
    ids, used = np.arange(6).reshape(B, 2), np.array([[512, 300], [1, 64], [500, 511]])
    q, k, v = (bf16(s * g.standard_normal((h, B, T, D))) for s, h in ((1.5, Hq), (1.0, Hkv), (1.0, Hkv)))
    got = pc.percache_attention_packed(0, q.reshape(Hq, B * T, D), k.reshape(Hkv, B * T, D), v.reshape(Hkv, B * T, D), np.arange(B + 1) * T, slot_ids=ids, used_len=used)[0]
    want = pc.percache_attention_reuse(0, *(x.transpose(0, 1).contiguous() for x in (q, k, v)), slot_ids=ids, used_len=used)
    torch.cuda.synchronize()
    got, want = host(got).reshape(B, T, Hq * D), host(want)
    assert np.linalg.norm(got - want) <= 2 * 3e-3 * np.linalg.norm(want) and np.abs(got - want).max() <= 2.0 ** -6 * float(host(v).max())
    pc.close()


def test_equal_calls_give_equal_bits():
    pc, g, kv, q, k, v, start, ids, used = build(SHAPES[6], "mixed")
    one = pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids, used_len=used, lse_out=True)
    two = pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids, used_len=used, lse_out=True)
    torch.cuda.synchronize()
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    pc.close()
