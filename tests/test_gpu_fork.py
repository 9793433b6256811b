"""Slots copied to slots through the C ABI: bits are compared."""
import numpy as np
import pytest
import torch

from oracle import packed_ref as ref
from paper_2601_11553_amd.binding import Percache

from gpu_util import DEV, bf16

pytestmark = pytest.mark.gpu


def filled(seed, Hkv, D, C, n, n8, lengths, n_layers=2):
    g = np.random.default_rng(seed)
    pc = Percache(n_layers=n_layers, hidden=64, n_q_heads=2 * Hkv, n_kv_heads=Hkv, head_dim=D, n_slots=n, slot_capacity=C, max_pos=512, n_slots_8bit=n8, device=DEV)
    for layer in range(n_layers):
        for s, m in enumerate(lengths if np.ndim(lengths) == 1 else lengths[layer]):
            if m:
                pc.percache_kv_put(layer, s, bf16(g.standard_normal((Hkv, m, D)) * 2.0 ** g.integers(-3, 4)), bf16(g.standard_normal((Hkv, m, D))))
    return pc, g


def contents(pc, layer):
    return {s: tuple(t.cpu() for t in pc.percache_kv_get(layer, s)) for s in range(pc.cfg.n_slots) if pc.percache_kv_len(layer, s)}


def check(pc, src, dst, n_tokens=None, layers=None):
    layer0, n_layers = layers or (0, pc.cfg.n_layers)
    want = []
    for layer in range(pc.cfg.n_layers):
        c = contents(pc, layer)
        want.append(ref.fork(c, src, dst, n_tokens) if layer0 <= layer < layer0 + n_layers else c)
    pc.percache_kv_fork(src, dst, n_tokens, layer0=layer0, n_layers=n_layers)
    torch.cuda.synchronize()
    for layer in range(pc.cfg.n_layers):
        got = contents(pc, layer)
        assert got.keys() == want[layer].keys()
        for s in got:
            assert all(torch.equal(a, b) for a, b in zip(got[s], want[layer][s])), (layer, s)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("formats", ["bf16", "8bit", "mixed"])
@pytest.mark.parametrize("length", [1, 63, 64, 65, 192])
def test_one_source_many_copies(D, formats, length):
    n = 12
    n8 = {"bf16": 0, "8bit": n, "mixed": 6}[formats]
    pc, g = filled(1, 2, D, 192, n, n8, [length] * 6 + [max(1, length - 1)] * 6)
    check(pc, [0, 0, 0, 6, 6], [1, 2, 5, 7, 11])
    pc.close()


@pytest.mark.parametrize("D,n8", [(64, 0), (128, 0), (128, 40), (64, 20)])
def test_any_map_of_slots(D, n8):
    """Permutations, chains, trees and rings with branches, lengths of any kind, some of the slots empty."""
    n, C = 40, 128
    for seed in range(6):
        g = np.random.default_rng(seed)
        lengths = g.integers(0, C + 1, n)
        pc, _ = filled(seed, 1, D, C, n, n8, lengths)
        halves = [range(n - n8), range(n - n8, n)]
        src, dst = [], []
        for half in halves:
            full = [s for s in half if lengths[s]]
            if not full:
                continue
            to = list(g.permutation(list(half))[:g.integers(1, len(half) + 1)])
            dst += to
            src += list(g.permutation(full)[:len(to)]) if seed % 2 and len(full) >= len(to) else list(g.choice(full, len(to)))
        order = g.permutation(len(src))
        src, dst = np.array(src)[order], np.array(dst)[order]
        cut = None if seed % 3 else np.array([g.integers(1, lengths[s] + 1) for s in src])
        check(pc, src, dst, cut)
        pc.close()


def test_swaps_rings_and_a_slot_cut_in_place():
    pc, g = filled(7, 2, 128, 128, 8, 0, [128, 5, 70, 64, 1, 100, 128, 3])
    check(pc, [0, 1], [1, 0])
    check(pc, [0, 1, 2, 3, 4], [1, 2, 3, 4, 0])
    check(pc, [2, 2, 5, 6], [2, 0, 6, 5], [3, 2, 60, 1])
    check(pc, [0], [0])
    pc.close()


def test_more_copies_than_a_launch_takes():
    """A ring of 600 slots, a chain of 300 behind each other and a source with 500 copies."""
    n = 1500
    g = np.random.default_rng(8)
    for D, n8 in ((64, 0), (64, n)):
        pc, _ = filled(8, 1, D, 64, n, n8, g.integers(1, 65, n), n_layers=1)
        ring, chain, star = np.arange(600), np.arange(600, 901), np.arange(901, 1402)
        check(pc, np.concatenate([np.roll(ring, 1), chain[:-1], np.full(500, 901)]), np.concatenate([ring, chain[1:], star[1:]]))
        pc.close()


def test_layers_of_different_lengths_and_a_range_of_layers():
    lengths = np.array([[5, 70, 128, 1], [5, 70, 128, 1], [64, 3, 9, 1], [5, 70, 127, 2]])
    pc, g = filled(9, 2, 64, 128, 4, 0, lengths, n_layers=4)
    check(pc, [0, 1], [3, 2], layers=(1, 2))
    check(pc, [2, 3, 0], [0, 2, 3])
    check(pc, [0, 1], [1, 0], n_tokens=[1, 1])
    check(pc, [], [])
    pc.close()


def test_padding_behind_the_last_token_is_zero():
    """A prefix of a slot whose later tokens are infinite: what reads whole blocks meets zeros behind it."""
    pc, g = filled(10, 2, 128, 64, 3, 0, [64, 0, 0], n_layers=1)
    k, v = pc.percache_kv_get(0, 0)
    v[:, 20:] = float("inf")
    pc.percache_kv_put(0, 0, k, v)
    pc.percache_kv_fork([0], [1], [20])
    q, kf, vf = (bf16(g.standard_normal((1, h, 3, 128))) for h in (4, 2, 2))
    out = pc.percache_attention_reuse(0, q, kf, vf, slot_ids=[[1]])
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    pc.close()


@pytest.mark.parametrize("D,n8", [(128, 0), (64, 0), (128, 3), (64, 3)])
def test_a_slot_cut_in_place_has_zeros_behind_its_last_token(D, n8):
    """The tokens that are cut off are infinite (8-bit: large); another slot takes them along before."""
    pc, g = filled(11, 2, D, 128, 3, n8, [100, 128, 7], n_layers=2)
    for layer in range(2):
        k, v = pc.percache_kv_get(layer, 0)
        v[:, 70:] = 2.0 ** 100 if n8 else float("inf")
        pc.percache_kv_put(layer, 0, k, v)
    check(pc, [0, 0, 1], [0, 2, 1], [70, 90, 64])
    for layer in range(2):
        q, kf, vf = (bf16(g.standard_normal((1, h, 3, D))) for h in (4, 2, 2))
        out = pc.percache_attention_reuse(layer, q, kf, vf, slot_ids=[[0, 1]])
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()
    pc.close()
