"""Bias, head norms and rotation of long packed batches, in every form that a launch takes (packed_shapes.py; test_packed_shapes.py says on the CPU which one that is).
Sampled rows against the float64 reference with the bounds of test_gpu_norm_rope.py; v, of all rows, is the fp32 sum of row and bias rounded once, to the bit."""
import numpy as np
import pytest
import torch

from oracle import packed_ref as ref

from gpu_util import DEV, bf16, host
from packed_shapes import ROWS
from test_gpu_norm_rope import EPS, THETA, context

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,D,rows", [r[:4] for r in ROWS])
def test_long_batches(Hq, Hkv, D, rows):
    g, gen = np.random.default_rng(rows), torch.Generator(device=DEV).manual_seed(rows)
    pc = context(Hq, Hkv, D, 5000)
    heads, F = Hq + 2 * Hkv, (Hq + 2 * Hkv) * D
    wide = (2 * torch.randn((rows, F + 40), generator=gen, device=DEV)).to(torch.bfloat16)
    x = wide[:, 8:8 + F]                       # rows at a distance
    axis = np.arange(D // 2) % 3
    pos = torch.randint(0, 5000, (3, rows), generator=gen, device=DEV, dtype=torch.int32)
    pos[:, 0], pos[:, -1] = 4999, 0
    q_norm, k_norm, bias = bf16(1 + 0.2 * g.standard_normal(D)), bf16(1 + 0.2 * g.standard_normal(D)), bf16(g.standard_normal(F))
    outs = dict(zip(("q_out", "k_out", "v_out"), (torch.full((h, rows, D), float("nan"), dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))))
    some = np.unique(np.concatenate([[0, 1, 2, rows - 2, rows - 1], g.integers(0, rows, 200)]))
    at = torch.from_numpy(some).to(DEV)
    f = lambda t: host(t).astype(np.float64)
    for b, qn, kn in ((bias, q_norm, k_norm), (None, None, k_norm)):
        q, k, v = pc.percache_qkv_norm_rope(x, pos, axis=axis, qkv_bias=b, q_norm=qn, k_norm=kn, eps=EPS, **outs)
        torch.cuda.synchronize()
        n = lambda t: None if t is None else f(t)
        wq, wk, _, qs, ks = ref.norm_rope(f(x[at]), Hq, Hkv, D, pos[:, at].cpu().numpy(), axis, THETA, n(b), n(qn), n(kn), EPS)
        for name, got, want, size in (("q", q, wq, qs), ("k", k, wk, ks)):
            err = np.abs(f(got[:, at]) - want) - 2.0 ** -8 * np.abs(want) - (D + 16) * 2.0 ** -24 * size
            assert err.max() <= 0, (name, err.max())
            assert torch.isfinite(got).all(), name      # (every row and head was written)
        vx = x.view(rows, heads, D)[:, Hq + Hkv:].transpose(0, 1)
        want_v = vx if b is None else (vx.float() + b.view(heads, 1, D)[Hq + Hkv:].float()).to(torch.bfloat16)
        assert torch.equal(v, want_v)
        for t in outs.values():
            t.fill_(float("nan"))
    pc.close()
