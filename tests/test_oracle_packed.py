"""Pins of the reference for packed prompts and several continuations (oracle/packed_ref.py)."""
import numpy as np
import pytest

from oracle import packed_ref as ref


def test_one_request_is_causal_attention():
    g = np.random.default_rng(1)
    Hq, Hkv, T, L, D = 4, 2, 7, 5, 16
    q, k, v = g.standard_normal((Hq, T, D)), g.standard_normal((Hkv, T, D)), g.standard_normal((Hkv, T, D))
    kc, vc = g.standard_normal((Hkv, L, D)), g.standard_normal((Hkv, L, D))
    out, lse, size, _ = ref.attend(q, k, v, kc, vc)
    for h in range(Hq):
        for i in range(T):
            keys, vals = np.concatenate([kc[h // 2], k[h // 2, :i + 1]]), np.concatenate([vc[h // 2], v[h // 2, :i + 1]])
            e = np.exp(keys @ q[h, i] / 4.0)
            assert np.allclose(out[i, h], e @ vals / e.sum()) and np.isclose(lse[h, i], np.log(e.sum()))
            assert (size[i, h] >= np.abs(out[i, h]) - 1e-12).all()


def test_rows_that_see_nothing_of_it_stay_as_they_are():
    g = np.random.default_rng(2)
    q, k, v = g.standard_normal((2, 6, 8)), g.standard_normal((2, 6, 8)), g.standard_normal((2, 6, 8))
    none = np.zeros((2, 0, 8))
    want = ref.attend(q, k, v, none, none)[0]
    k[:, 4], v[:, 4] = np.nan, np.inf
    assert np.allclose(ref.attend(q, k, v, none, none)[0][:4], want[:4])


def test_a_turn_keeps_lengths_and_relative_positions():
    g = np.random.default_rng(3)
    D = 32
    x = g.standard_normal((3, 3 * D))
    axis = np.arange(D // 2) % 3
    pos = g.integers(0, 500, (3, 3))
    q, k, v, _, _ = ref.norm_rope(x, 1, 1, D, pos, axis, 1e4)
    assert np.allclose(np.linalg.norm(q[0], axis=1), np.linalg.norm(x[:, :D], axis=1)) and np.array_equal(v[0], x[:, 2 * D:])
    q2, k2, _, _, _ = ref.norm_rope(x, 1, 1, D, pos + np.array([[17], [5], [9]]), axis, 1e4)
    assert np.allclose((q * k).sum(-1), (q2 * k2).sum(-1)) and np.allclose(q[0] @ k[0].T, q2[0] @ k2[0].T)
    # position 0 turns nothing, and the first pair of axis 0 turns by the position itself
    assert np.allclose(ref.norm_rope(x, 1, 1, D, pos * 0, axis, 1e4)[0][0], x[:, :D])
    z = np.zeros((1, 3 * D))
    z[0, 0] = 1.0
    assert np.allclose(ref.norm_rope(z, 1, 1, D, np.array([[2], [7], [8]]), axis, 1e4)[0][0, 0, [0, D // 2]], [np.cos(2), np.sin(2)])


def test_head_norm():
    g = np.random.default_rng(4)
    x, gain = g.standard_normal((5, 3 * 16)), g.standard_normal(16)
    q = ref.norm_rope(x, 1, 1, 16, np.zeros((1, 5), int), np.zeros(8, int), 1e4, q_norm=gain, eps=0.0)[0][0]
    assert np.allclose((q / gain) ** 2 @ np.ones(16), 16.0)


@pytest.mark.parametrize("best", [1, 4, 30])
def test_selection_is_a_sort_of_all_candidates(best):
    g = np.random.default_rng(5)
    x, s = g.integers(-3, 4, (3, 4, 6)).astype(float), g.integers(-2, 1, (3, 4)).astype(float)
    x[0, 1] = x[0, 0]
    s[0, 1] = s[0, 0]
    s[1, 2] = -np.inf
    x[2, 0, :4] = -np.inf
    parent, token, score = ref.beams(x, s, best)
    for b in range(3):
        with np.errstate(divide="ignore"):
            t = (s[b][:, None] + x[b] - np.log(np.exp(x[b]).sum(1))[:, None]).ravel()
        order = [c for c in np.argsort(-t, kind="stable") if np.isfinite(t[c])][:best]
        # (equal sums of different terms may differ in the last place; what is compared is the score and, where scores differ, the place)
        assert np.allclose(score[b, :len(order)], t[order]) and (parent[b, len(order):] == -1).all()
        assert np.allclose(t[parent[b, :len(order)] * 6 + token[b, :len(order)]], score[b, :len(order)])
        pairs = list(zip(-np.round(score[b, :len(order)], 9), parent[b], token[b]))
        assert pairs == sorted(pairs) and len(set(pairs)) == len(pairs)


def test_copies_take_what_was_there_before():
    one = {i: (np.full((1, 3, 2), i), np.full((1, 3, 2), 10 + i)) for i in range(4)}
    got = ref.fork(dict(one), [0, 1, 2, 0], [1, 2, 0, 3], [3, 2, 1, 3])
    assert [int(got[i][0][0, 0, 0]) for i in range(4)] == [2, 0, 1, 0] and [got[i][0].shape[1] for i in range(4)] == [1, 3, 2, 3]
