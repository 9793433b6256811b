"""Projection of drafted nodes in every form that the calls take by size, each row against float64.

Bound: a feature is an fp32 sum of K products of bf16 numbers, off by at most (K + 4) 2^-24 of the sum of their sizes; the rotation takes two of them with
table entries rounded to fp32 (2^-24 each, and the products and their sum: 4 more); one rounding to bf16, 2^-8 of the result."""
import numpy as np
import pytest
import torch

from oracle import draft_ref as ref
from paper_2601_11553_amd.binding import Percache

from gpu_util import DEV
from test_gpu_draft import random_tree

pytestmark = pytest.mark.gpu

# form (on 256 CUs), hidden, query heads, kv heads, head size, queries, nodes of each
FORMS = [
    # tiles of 128 nodes with every stage requested ahead: contractions shorter than the ring of four stages and longer, row counts around a tile's, an
    # odd number of heads, exactly as many tiles as CUs
    ("deep", 64, 72, 8, 128, 3, 43), ("deep", 128, 72, 8, 128, 1, 192), ("deep", 192, 72, 8, 128, 2, 97), ("deep", 256, 72, 8, 128, 1, 255), ("deep", 320, 72, 8, 128, 1, 256),
    ("deep", 2048, 32, 8, 128, 8, 63), ("deep", 2048, 32, 8, 128, 3, 171), ("deep", 1024, 3, 1, 128, 5, 231), ("deep", 4160, 2, 1, 128, 1, 254), ("deep", 64, 3, 1, 128, 9, 128),
    ("deep", 64, 14, 2, 64, 5, 206), ("deep", 128, 14, 2, 64, 8, 129), ("deep", 192, 2, 1, 64, 5, 230), ("deep", 4096, 14, 2, 64, 2, 150), ("deep", 320, 48, 8, 64, 4, 256),
    # one tile more than CUs, and other counts that leave them the one-head tiles of 64, 128 and 192 nodes
    ("plain 2", 320, 48, 8, 64, 5, 205), ("plain 1", 64, 256, 8, 64, 1, 150), ("plain 3", 128, 48, 8, 64, 10, 210),
    ("plain 1", 64, 120, 8, 128, 3, 50), ("plain 2", 256, 32, 8, 128, 4, 175), ("plain 3", 128, 35, 7, 128, 6, 225),
    # two-head tiles of 192, 256 and 320 nodes
    ("wide 3", 512, 8, 2, 128, 8, 200), ("wide 4", 768, 16, 4, 128, 20, 210), ("wide 5", 512, 16, 4, 128, 24, 225),
    # few rows
    ("few", 512, 4, 2, 128, 1, 1), ("few", 1024, 16, 8, 128, 3, 60), ("few", 256, 14, 2, 64, 2, 128),
]


def project(form, H, Hq, Hkv, D, B, T):
    g = np.random.default_rng(T + H)
    max_pos = 700
    pc = Percache(n_layers=1, hidden=H, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, n_slots=1, slot_capacity=64, max_pos=max_pos, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(T + H)
    x = torch.randn((B, T, H), generator=gen, device=DEV).bfloat16()
    w = (0.02 * torch.randn(((Hq + 2 * Hkv) * D, H), generator=gen, device=DEV)).bfloat16()
    parents = [random_tree(g, T, max(1, T - b % 3)) for b in range(B)]
    depth = np.array([ref.depths(p) for p in parents])
    pos0 = np.array([int(g.integers(0, max_pos - d.max())) for d in depth])
    pos0[-1] = max_pos - 1 - depth[-1].max()   # (the deepest node of the last query at the last position)
    return pc, x, w, parents, pos0, torch.from_numpy(pos0[:, None] + depth).to(DEV)


@pytest.mark.parametrize("form,H,Hq,Hkv,D,B,T", FORMS)
def test_projection_in_every_form(form, H, Hq, Hkv, D, B, T):
    pc, x, w, parents, pos0, pos = project(form, H, Hq, Hkv, D, B, T)
    q, k, v = pc.percache_qkv_rope_draft(x, w, pos0, parents=parents)
    torch.cuda.synchronize()
    x64, w64 = x.double().view(B * T, H), w.double()
    heads = lambda y: y.view(B, T, Hq + 2 * Hkv, D).transpose(1, 2)   # noqa: E731
    y, size = heads(torch.mm(x64, w64.t().contiguous())), heads(torch.mm(x64.abs(), w64.abs().t().contiguous()))
    angle = pos.double()[:, None, :, None] * 10000.0 ** (-2.0 * torch.arange(D // 2, device=DEV, dtype=torch.float64) / D)
    cos, sin = angle.cos(), angle.sin()

    def turned(y, sign):
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([a * cos - sign * b * sin, b * cos + a * sin], -1)
    for name, got, at in (("q", q, slice(0, Hq)), ("k", k, slice(Hq, Hq + Hkv)), ("v", v, slice(Hq + Hkv, None))):
        want, s = y[:, at], size[:, at]
        if name != "v":
            want = turned(want, 1.0)
            s = torch.cat([s[..., :D // 2] + s[..., D // 2:]] * 2, -1)
        err = (got.double() - want).abs() - 2.0 ** -8 * want.abs() - (1 + 2.0 ** -8) * (H + 8) * 2.0 ** -24 * s
        assert err.max() <= 0, (name, float(err.max()), tuple(int(i) for i in np.unravel_index(int(err.argmax()), err.shape)))
    pc.close()
