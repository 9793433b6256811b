"""Selection over beams and vocabulary through the C ABI against the float64 reference: tokens and parents have to be equal, scores to a few roundings.

Bound of a score: the sum of exponentials is off by about 2^-22 of itself (each term's exponent by |x - max| 2^-24, weighed by the term; sums in fp32 of at
most a few hundred terms a lane, in 64 bits above), the score is formed in 64 bits and rounded once: 2^-21 + 2^-23 |score|.  Inputs whose
candidates of different beams lie closer than that are not used where the order is compared: the references' gaps are looked at."""
import numpy as np
import pytest
import torch

from oracle import packed_ref as ref
from paper_2601_11553_amd.binding import Percache

from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pc():
    pc = Percache(n_slots=1, slot_capacity=64, max_pos=64, device=DEV)
    yield pc
    pc.close()


def check(pc, logits, scores, best):
    parent, token, score = pc.percache_beam_select(logits, scores, best)
    torch.cuda.synchronize()
    wp, wt, ws = ref.beams(logits.double().cpu().numpy(), scores.double().cpu().numpy(), best)
    gp, gt, gs = (x.cpu().numpy() for x in (parent, token, score))
    live = wp >= 0
    assert (gp[~live] == -1).all() and (gt[~live] == -1).all() and (gs[~live] == -np.inf).all()
    assert (np.abs(gs[live].astype(np.float64) - ws[live]) <= 2.0 ** -21 + 2.0 ** -23 * np.abs(ws[live])).all()
    assert np.array_equal(gp, wp) and np.array_equal(gt, wt), np.argwhere((gp != wp) | (gt != wt))[:5]
    return parent, token, score


def drawn(seed, batch, beams, vocab, dtype, scale=2.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = (torch.randn((batch, beams, vocab), generator=g, device=DEV) * scale).to(dtype)
    return x, -10 * torch.rand((batch, beams), generator=g, device=DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,beams,vocab,best", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 7, 4), (1, 4, 32000, 8), (3, 8, 4097, 16), (2, 16, 50001, 32), (5, 1, 2047, 1), (2, 2, 16384, 64),
                                                   (70, 4, 999, 8), (1, 2, 150001, 3), (2, 64, 300, 32), (1, 32, 8000, 64)])
def test_any_sizes(pc, dtype, batch, beams, vocab, best):
    check(pc, *drawn(batch + vocab, batch, beams, vocab, dtype), best)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_equal_logits_go_by_token_and_equal_beams_by_beam(pc, dtype):
    """All logits alike, a few values over and over, whole beams alike."""
    for vocab in (3, 64, 5000, 40000):
        x = torch.zeros((2, 3, vocab), dtype=dtype, device=DEV)
        x[1] = (torch.arange(vocab, device=DEV) * 7 % 5).to(dtype)
        check(pc, x, torch.zeros((2, 3), device=DEV), 12)
    x, s = drawn(5, 1, 1, 9000, torch.bfloat16, 1.0)
    check(pc, x.expand(1, 6, 9000).contiguous().to(dtype), s.expand(1, 6).contiguous(), 20)
    # the best ones at the end, one above the other, and signed zeros (equal)
    x = torch.arange(20000, device=DEV, dtype=torch.float32).div_(2000).view(1, 1, -1).to(dtype)
    check(pc, x, torch.zeros((1, 1), device=DEV), 64)
    x = torch.full((1, 2, 3000), -1.0, dtype=dtype, device=DEV)
    x[0, :, 100::50], x[0, :, 101::50] = 0.0, -0.0
    check(pc, x, torch.zeros((1, 2), device=DEV), 30)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forbidden_tokens_dead_beams_and_numbers_that_are_none(pc, dtype):
    x, s = drawn(6, 6, 4, 6000, dtype)
    x[0] = -float("inf")                    # nothing is allowed
    x[1, :, 3:] = -float("inf")             # three tokens a beam
    x[1, 2, :] = -float("inf")
    x[2, 0, 17] = float("nan")              # (the beam is out)
    x[2, 1, 5999] = float("inf")
    s[3] = -float("inf")                    # no beam at all
    s[4, 1:] = -float("inf")                # a first step
    s[4, 0] = 0.0
    s[5, 1], s[5, 2] = float("nan"), float("inf")
    x[5, 0, :5000] = -float("inf")
    check(pc, x, s, 16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_at_a_distance_and_at_odd_places(pc, dtype):
    """Rows that start at any place of their 16 bytes: a view into a wider tensor."""
    wide, s = drawn(8, 2, 3, 3013, dtype)
    for lo, n in ((0, 3013), (1, 3001), (3, 2999), (7, 8), (5, 3), (2, 1), (6, 2050)):
        check(pc, wide[:, :, lo:lo + n], s, min(4, n))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_many_rounds(pc, dtype):
    """So many rows that each is cut into few stretches and a lane has logits from several rounds: its best ones in one of them, in all, alike or nowhere."""
    x, s = drawn(12, 48, 8, 50000, dtype)
    x[1] = torch.sort(x[1], -1)[0]
    for first, step in ((5, 1024), (7, 2048)):
        n = x[2, :, first::step].shape[1]
        x[2, :, first::step] = (20 + 0.25 * torch.arange(n, device=DEV) * (1 if first == 5 else -1)).to(dtype)
        x[3, :, first::step] = 18
    x[4, :, :] = -float("inf")
    x[4, 3, ::4099] = 1.0
    x[5] = -3.0
    x[6, :, :20000] = -float("inf")
    x[7, :, 256:] = x[7, :, 256:].clamp_(max=6)
    x[7, :, :256] = torch.linspace(9, 10, 256, device=DEV).to(dtype)
    s[1:8] = 0.0
    s[1:8, 1:] = -5.0 * torch.arange(1, 8, device=DEV)
    check(pc, x, s, 16)


def test_large_and_small_logits(pc):
    x, s = drawn(9, 2, 2, 5000, torch.float32)
    check(pc, x * 40, s, 8)
    check(pc, x * 1e-3, s, 8)
    x[0, 0, 7], x[0, 1, 9] = 3e38, 1e30
    check(pc, x, s, 2)


def test_two_streams_at_once(pc):
    """The binding keeps a workspace for each stream."""
    sets = [drawn(20 + i, 4, 4, 30000, torch.bfloat16) for i in range(2)]
    want = [pc.percache_beam_select(x, s, 8) for x, s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for (x, s), st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(pc.percache_beam_select(x, s, 8))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(r, want[i % 2]))
