"""Packed attention where blocks stay tall (256 or 128 stacked rows): the shapes of packed_shapes.py, of which test_packed_shapes.py says on the CPU which blocks,
partitions and formats they plan.  Reference and bounds are those of test_gpu_packed.py:
|error| <= (2^-7 + 2^-13) sum_j p_j |v_j|, log-sum-exp (D S + n + 8 |lse| + 64) 2^-24."""
import numpy as np
import pytest
import torch

from oracle import packed_ref as ref

from gpu_util import DEV, host
from packed_shapes import CALLS, MIDDLE, RUBBISH, RUBBISH_CALLS, TALL, slots_of
from test_gpu_draft import cached, make, stored
from test_gpu_packed import packed

pytestmark = pytest.mark.gpu
SHAPES = {**TALL, **MIDDLE}


class Case:
    """A call's inputs and, once, what its rows have to be."""

    def __init__(self, shape, formats, seed=71, gap=(0, 0), spoil=None, scale=1.0):
        Hq, Hkv, D, T, _, C = shape
        tokens, self.ids, self.used = slots_of(shape)
        self.pc, self.g, self.kv = make(seed, Hq, Hkv, D, C, formats, tokens, max_pos=16384)
        self.start = gap[0] + np.concatenate([[0], np.cumsum(T)])
        self.q, self.k, self.v = packed(self.g, Hq, Hkv, D, int(self.start[-1]) + gap[1])
        self.q = self.q * scale
        self.skip = set()
        qh, kh, vh = (host(x).astype(np.float64) for x in (self.q, self.k, self.v))
        if spoil:
            spoil(self)
        self.want = []
        for s in range(len(T)):
            a, b = int(self.start[s]), int(self.start[s + 1])
            kc, vc = cached(self.kv, self.ids[s], self.used[s]) if self.ids is not None else cached(self.kv, [], [])
            self.want.append((a, b, D * 1.0, kc.shape[1], *ref.attend(qh[:, a:b], kh[:, a:b], vh[:, a:b], kc, vc)))

    def run(self, n_splits=0):
        Hq, N, D = self.q.shape
        out = torch.full((N, Hq * D), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((Hq, N), 7.0, dtype=torch.float32, device=DEV)
        n_splits = min(n_splits, self.pc.lib.percache_packed_max_splits(self.pc.ctx, len(self.start) - 1, N))
        self.pc.percache_attention_packed(0, self.q, self.k, self.v, self.start, slot_ids=self.ids, used_len=self.used, attn_out=out, lse_out=lse, n_splits=n_splits)
        torch.cuda.synchronize()
        return out, lse

    def check(self, n_splits=0):
        Hq, N, D = self.q.shape
        out, lse = self.run(n_splits)
        o, ls = host(out).astype(np.float64).reshape(N, Hq, D), lse.double().cpu().numpy()
        mine = np.zeros(N, bool)
        for s, (a, b, d, n, want, wl, size, S) in enumerate(self.want):
            mine[a:b] = True
            rows = [i for i in range(b - a) if a + i not in self.skip]
            got, gl = o[a:b], ls[:, a:b]
            assert np.isfinite(got[rows]).all() and np.isfinite(gl[:, rows]).all(), (s, np.argwhere(~np.isfinite(got[rows]))[:5])
            err = (np.abs(got - want) - (2.0 ** -7 + 2.0 ** -13) * size)[rows]
            assert err.max() <= 0, (s, a, b, err.max(), np.argwhere(err > 0)[:5], (err > 0).sum())
            tol = (d * S + n + b - a + 8 * np.abs(wl) + 64) * 2.0 ** -24
            assert (np.abs(gl - wl) <= tol)[:, rows].all(), (s, np.abs(gl - wl)[:, rows].max())
        assert (o[~mine] == 7).all() and (ls[:, ~mine] == 7).all()
        return out, lse


GROUPS = {}
for c in CALLS:
    GROUPS.setdefault(c[:2], []).append(c[2])


@pytest.mark.parametrize("name,formats", list(GROUPS), ids=["-".join(x) for x in GROUPS])
def test_tall_blocks(name, formats):
    case = Case(SHAPES[name], formats)
    for n_splits in GROUPS[name, formats]:
        print(name, formats, n_splits, flush=True)
        case.check(n_splits)
    case.pc.close()


@pytest.mark.parametrize("name", ["32over32x64", "32over8x128"])
def test_rows_of_nobody_beside_tall_blocks(name):
    """They hold NaN: nothing reads or writes them."""
    def spoil(c):
        for x in (c.q, c.k, c.v):
            x[:, :int(c.start[0])] = float("nan")
            x[:, int(c.start[-1]):] = float("nan")
    case = Case(SHAPES[name], "bf16", gap=(13, 70), spoil=spoil)
    for n_splits in (0, 2):
        case.check(n_splits)
    case.pc.close()


def later_rows(c):
    """Some rows' K and V are infinite or NaN: rows from there on are not looked at, those before them have to be what they are without it."""
    for s in range(len(c.start) - 1):
        T = int(c.start[s + 1] - c.start[s])
        for i, kx, vx in ((T - 1, float("nan"), float("inf")), (T * 3 // 4, float("inf"), -float("inf")), (T // 2, 2.0, float("nan")))[:1 + s % 3] if T > 40 else ():
            row = int(c.start[s]) + i
            c.k[:, row], c.v[:, row] = kx, vx
            c.v[:, row, 1::2] = 1.0
            c.skip |= set(range(row, int(c.start[s + 1])))


@pytest.mark.parametrize("name", list(RUBBISH))
@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
def test_rubbish_in_later_rows_of_tall_blocks(name, formats):
    case = Case(RUBBISH[name], formats, seed=72, spoil=later_rows)
    for n_splits in [n for x, f, n in RUBBISH_CALLS if (x, f) == (name, formats)]:
        print(name, formats, n_splits, flush=True)
        case.check(n_splits)
    case.pc.close()


@pytest.mark.parametrize("name", list(RUBBISH))
def test_rubbish_behind_used_lengths_of_tall_blocks(name):
    """Tokens of a slot behind the used length are infinite or NaN (bf16 slots)."""
    def spoil(c):
        for row, use in zip(c.ids, c.used):
            for s, n in zip(row, use):
                k, v = c.pc.percache_kv_get(0, int(s))
                if n < k.shape[1]:
                    k[:, n:], v[:, n:] = float("nan"), float("inf")
                    v[:, n + 1:, ::3] = float("nan")
                    c.pc.percache_kv_put(0, int(s), k, v)
        c.kv = stored(c.pc)
    case = Case(RUBBISH[name], "bf16", seed=73, spoil=spoil)
    for n_splits in (0, 1, 3):
        case.check(n_splits)
    case.pc.close()


@pytest.mark.parametrize("name", ["32over8x128", "14over2x64"])
def test_infinite_values_that_rows_of_tall_blocks_see(name):
    """V infinite in one dimension of one token: infinite there for every row that sees it, within the bound of the finite call elsewhere."""
    case = Case(RUBBISH[name], "bf16", seed=74)
    Hq, N, D = case.q.shape
    marks = [(0, 1, 5), (0, 290, 11), (2, 0, 9), (2, 255, 3), (2, 511, 40)]
    for s, i, d in marks:
        case.v[:, int(case.start[s]) + i, d] = float("inf")
    for n_splits in (0, 1, 3):
        got = host(case.run(n_splits)[0]).astype(np.float64).reshape(N, Hq, D)
        for s, (a, b, _, _, want, _, size, _) in enumerate(case.want):
            hit = np.zeros((b - a, Hq, D), bool)
            for r, i, d in marks:
                if r == s:
                    hit[i:, :, d] = True
            assert (got[a:b][hit] == np.inf).all()
            assert (np.abs(got[a:b] - want) <= (2.0 ** -7 + 2.0 ** -13) * size)[~hit].all(), (s, n_splits)
    case.pc.close()


@pytest.mark.parametrize("name", ["32over8x128", "32over32x64"])
def test_peaked_rows_of_tall_blocks(name):
    """Scores of +-100 and more: the reference exponent moves in the middle of a walk."""
    case = Case(SHAPES[name], "mixed", seed=75, scale=8.0)
    for n_splits in (0, 2):
        case.check(n_splits)
    case.pc.close()
