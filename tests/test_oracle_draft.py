"""Pins of the float64 reference for drafted tokens and eviction inside a slot (oracle/draft_ref.py)."""
import itertools

import numpy as np
import pytest

import oracle
from oracle import draft_ref as ref


def test_ancestors_and_depths_of_a_small_tree():
    parents = [-1, 0, 0, 1, -1, 4, -2, 3]
    assert ref.ancestors(parents) == [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {4}, {4, 5}, set(), {0, 1, 3, 7}]
    assert ref.depths(parents) == [0, 1, 1, 2, 0, 1, 0, 3]


def test_a_plain_sequence_is_causal_attention():
    g = np.random.default_rng(0)
    Hq, Hkv, T, D, C = 4, 2, 7, 64, 64
    q, kd, vd = g.standard_normal((Hq, T, D)), g.standard_normal((Hkv, T, D)), g.standard_normal((Hkv, T, D))
    store_k, store_v = g.standard_normal((1, Hkv, C, D)), g.standard_normal((1, Hkv, C, D))
    out, lse, _, _, probs = ref.attend(q, store_k[0, :, :19], store_v[0, :, :19], kd, vd, ref.ancestors([i - 1 for i in range(T)]))
    want = oracle.attention_reuse(q.astype(np.float32), kd.astype(np.float32), vd.astype(np.float32), store_k.astype(np.float32), store_v.astype(np.float32), [0], [19])
    assert np.abs(out.reshape(T, Hq * D) - want).max() < 1e-5
    for p, nodes in probs.values():
        assert abs(p.sum() + sum(nodes.values()) - 1) < 1e-12
    cached, draft = ref.weights(probs, Hq, Hkv, T, 19, [0, 3, 3])
    assert abs(cached.sum() + draft.sum() - 3 * Hq) < 1e-9


def test_a_branch_does_not_see_its_sibling():
    g = np.random.default_rng(1)
    q, kd, vd = g.standard_normal((2, 3, 64)), g.standard_normal((1, 3, 64)), g.standard_normal((1, 3, 64))
    none = np.zeros((1, 0, 64))
    a = ref.attend(q, none, none, kd, vd, ref.ancestors([-1, 0, 0]))[0]
    vd[:, 1], kd[:, 1] = 1e3, 7.0
    b = ref.attend(q, none, none, kd, vd, ref.ancestors([-1, 0, 0]))[0]
    assert np.array_equal(a[2], b[2]) and not np.array_equal(a[1], b[1])
    assert np.allclose(a[0, :], vd[0, 0])


@pytest.mark.parametrize("have,n_keep,n_first,n_last", [(7, 3, 0, 0), (7, 4, 1, 1), (7, 5, 2, 3), (6, 6, 0, 0), (5, 9, 1, 1)])
def test_keep_takes_the_largest_sum_of_weights_first_of_ties(have, n_keep, n_first, n_last):
    g = np.random.default_rng(have * 10 + n_keep)
    for _ in range(20):
        w = g.integers(0, 3, have).astype(float)
        got = ref.keep(w, have, n_keep, n_first, n_last)
        if have <= n_keep:
            assert got == list(range(have))
            continue
        fixed = set(range(n_first)) | set(range(have - n_last, have))
        choices = [c for c in itertools.combinations(range(have), n_keep) if fixed <= set(c)]
        best = max(sum(w[list(c)]) for c in choices)
        assert tuple(got) == min(c for c in choices if sum(w[list(c)]) == best)   # (in order: the earlier of equal ones)


def test_keep_puts_nan_last_and_infinities_in_order():
    w = [np.nan, 1.0, -np.inf, np.inf, 0.0, np.nan]
    assert ref.keep(w, 6, 3, 0, 0) == [1, 3, 4]
    assert ref.keep(w, 6, 5, 0, 0) == [0, 1, 2, 3, 4]
