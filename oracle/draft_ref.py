"""Reference for drafted tokens and for eviction inside a slot, in float64 numpy.  TEST INFRASTRUCTURE ONLY.

Everything is written from the definitions, one query, head and row at a time; parity unpinned by the paper (it names
neither operator), pinned by tests/test_oracle_draft.py: a plain sequence is the ordinary causal attention, every row's
weights sum to one, eviction agrees with a brute-force sort.
"""
from __future__ import annotations

import math

import numpy as np


def ancestors(parents):
    """For each node the set of nodes it looks at (itself included), empty for padding (-2)."""
    seen = []
    for i, p in enumerate(parents):
        seen.append(set() if p == -2 else {i} | (seen[p] if p >= 0 else set()))
    return seen


def depths(parents):
    d = []
    for p in parents:
        d.append(d[p] + 1 if p >= 0 else 0)
    return d


def attend(q, k_cached, v_cached, k_draft, v_draft, seen):
    """One query.  q [Hq, T, D]; k_cached, v_cached [Hkv, L, D]; k_draft, v_draft [Hkv, T, D]; seen: ancestors().
    Returns out [T, Hq, D], lse [Hq, T], a bound of the size of what is added up (sum of p |v|) [T, Hq, D], the largest sum of |q_d k_d| / sqrt(D)
    of any score, and the probabilities as {(head, row): (over the cached keys, {node: p})}."""
    Hq, T, D = q.shape
    Hkv, L, _ = k_cached.shape
    out, size = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse = np.full((Hq, T), -np.inf)
    probs, largest = {}, 0.0
    for h in range(Hq):
        g = h // (Hq // Hkv)
        for i in range(T):
            nodes = sorted(seen[i])
            if not nodes:
                probs[h, i] = (np.zeros(L), {})
                continue
            keys = np.concatenate([k_cached[g], k_draft[g, nodes]])
            vals = np.concatenate([v_cached[g], v_draft[g, nodes]])
            s = keys @ q[h, i] / math.sqrt(D)
            largest = max(largest, float((np.abs(keys) @ np.abs(q[h, i])).max()) / math.sqrt(D))
            top = s.max()
            lse[h, i] = top + math.log(np.exp(s - top).sum())
            p = np.exp(s - lse[h, i])
            out[i, h], size[i, h] = p @ vals, p @ np.abs(vals)
            probs[h, i] = (p[:L], dict(zip(nodes, p[L:])))
    return out, lse, size, largest, probs


def weights(probs, Hq, Hkv, T, L, rows):
    """What the rows (with repetition) of one query pay: (cached [Hkv, L], draft [Hkv, T])."""
    cached, draft = np.zeros((Hkv, L)), np.zeros((Hkv, T))
    for h in range(Hq):
        g = h // (Hq // Hkv)
        for i in rows:
            p, nodes = probs[h, i]
            cached[g] += p
            for j, x in nodes.items():
                draft[g, j] += x
    return cached, draft


def keep(w, have, n_keep, n_first, n_last):
    """Indexes that one head keeps of a slot's first `have` tokens with weights w."""
    if have <= n_keep:
        return list(range(have))
    fixed = [t for t in range(have) if t < n_first or t >= have - n_last]
    rest = [t for t in range(have) if n_first <= t < have - n_last]
    rank = sorted(rest, key=lambda t: (math.isnan(w[t]), -w[t] if not math.isnan(w[t]) else 0.0, t))
    return sorted(fixed + rank[:n_keep - len(fixed)])
