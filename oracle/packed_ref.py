"""Reference for packed prompts and for several continuations of one, in float64 numpy.  TEST INFRASTRUCTURE ONLY.

Everything is written from the definitions; parity unpinned by the paper (it names none of these operators), pinned by
tests/test_oracle_packed.py: one request is the ordinary causal attention, a turn keeps lengths and relative positions, a
selection agrees with a sort of all candidates.
"""
from __future__ import annotations

import math

import numpy as np


def attend(q, k, v, k_cached, v_cached):
    """One request.  q [Hq, T, D]; k, v [Hkv, T, D]; k_cached, v_cached [Hkv, L, D].  Row i sees the L cached keys and rows 0..i.
    Returns out [T, Hq, D], lse [Hq, T], a bound of what is added up (sum of p |v|) [T, Hq, D] and the largest sum of |q_d k_d| / sqrt(D) of a score.
    What a row does not see is not touched (it need not be finite)."""
    Hq, T, D = q.shape
    L = k_cached.shape[1]
    out, size, lse, largest = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((Hq, T)), 0.0
    for h in range(Hq):
        g = h // (Hq // k.shape[0])
        keys, vals = np.concatenate([k_cached[g], k[g]]), np.concatenate([v_cached[g], v[g]])
        with np.errstate(invalid="ignore", over="ignore"):
            s = q[h] @ keys.T / math.sqrt(D)
            bound = np.abs(q[h]) @ np.abs(keys).T / math.sqrt(D)
        sees = np.arange(L + T)[None, :] <= L + np.arange(T)[:, None]
        largest = max(largest, float(np.where(sees, bound, 0.0).max()))
        s = np.where(sees, s, -np.inf)
        top = s.max(1)
        lse[h] = top + np.log(np.exp(s - top[:, None]).sum(1))
        p = np.exp(s - lse[h][:, None])
        if np.isfinite(vals).all():
            out[:, h], size[:, h] = p @ vals, p @ np.abs(vals)
        else:
            for i in range(T):
                with np.errstate(invalid="ignore"):
                    out[i, h] = (p[i, :L + i + 1, None] * vals[:L + i + 1]).sum(0)
                    size[i, h] = (p[i, :L + i + 1, None] * np.abs(vals[:L + i + 1])).sum(0)
    return out, lse, size, largest


def norm_rope(x, Hq, Hkv, D, pos, axis, theta, bias=None, q_norm=None, k_norm=None, eps=1e-6):
    """x [N, (Hq + 2 Hkv) * D]; pos [axes, N]; axis [D/2].  Returns q, k, v by heads and, for q and k, the size |a| + |b| of what a turn adds up."""
    N = x.shape[0]
    y = (x + (0 if bias is None else bias)).reshape(N, Hq + 2 * Hkv, D).transpose(1, 0, 2).astype(np.float64)
    q, k, v = y[:Hq], y[Hq:Hq + Hkv], y[Hq + Hkv:]
    if q_norm is not None:
        q = q / np.sqrt((q * q).mean(-1, keepdims=True) + eps) * q_norm
    if k_norm is not None:
        k = k / np.sqrt((k * k).mean(-1, keepdims=True) + eps) * k_norm
    m = np.arange(D // 2)
    angle = pos[np.asarray(axis), :].T.astype(np.float64) * theta ** (-2.0 * m / D)       # [N, D/2]

    def turn(z):
        w = (z[..., :D // 2] + 1j * z[..., D // 2:]) * np.exp(1j * angle)
        size = np.abs(z[..., :D // 2]) + np.abs(z[..., D // 2:])
        return np.concatenate([w.real, w.imag], -1), np.concatenate([size, size], -1)
    (q, q_size), (k, k_size) = turn(q), turn(k)
    return q, k, v, q_size, k_size


def beams(logits, scores, best):
    """logits [B, N, V], scores [B, N] (float64).  Returns parent, token (int64) and score (float64), each [B, best]."""
    B, N, V = logits.shape
    parent, token, score = np.full((B, best), -1), np.full((B, best), -1), np.full((B, best), -np.inf)
    for b in range(B):
        found = []
        for i in range(N):
            x = logits[b, i]
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                top = x.max()
                lse = top + np.log(np.exp(x - top).sum())
            if not (np.isfinite(lse) and np.isfinite(scores[b, i])):
                continue
            total = scores[b, i] - lse + x
            ok = np.flatnonzero(x > -np.inf)
            found += [(-total[t], i, int(t)) for t in ok[np.lexsort((ok, -x[ok]))[:best]]]
        for r, (z, i, t) in enumerate(sorted(found)[:best]):
            parent[b, r], token[b, r], score[b, r] = i, t, -z
    return parent, token, score


def fork(slots, src, dst, n_tokens=None):
    """slots: {id: (k, v)} with k, v [Hkv, tokens, D]; the copies of a call, all from what the slots held before it."""
    old = dict(slots)
    for j, (s, d) in enumerate(zip(src, dst)):
        n = old[s][0].shape[1] if n_tokens is None else n_tokens[j]
        slots[d] = tuple(x[:, :n] for x in old[s])
    return slots
