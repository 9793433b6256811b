"""Decoding by verified drafts over a bounded cache, one layer: per step every query drafts a tree of tokens, the tree is projected and attended over
[retrieved chunks ; the query's own slot ; the tree] in one call each, the accepted path pays its attention weights and moves into the query's slot, and
a slot that has reached its budget is cut to the tokens that drew the most weight.

Hidden states, weights and the choice of the accepted path are random here (drafting and accepting take a model's logits); the data flow is that
of a serving loop.  Run it on the GPU:  python examples/draft_decode.py [--steps N] [--batch B] [--nodes T]
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2601_11553_amd.binding import Percache  # noqa: E402


class DraftDecoder:
    """Slots 0 .. chunks - 1: the retrieved chunks, which all queries share; slot chunks + b: query b's own tokens."""

    def __init__(self, batch=4, nodes=16, chunks=4, capacity=256, budget=192, hidden=1024, heads=16, kv_heads=8, head_dim=128, first=4, last=32, seed=0,
                 n_slots_8bit=0, device="cuda:0"):
        self.batch, self.nodes, self.chunks, self.budget, self.first, self.last = batch, nodes, chunks, budget, first, last
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.pc = Percache(n_layers=1, hidden=hidden, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, n_slots=chunks + batch, slot_capacity=capacity,
                           max_pos=1 << 15, n_slots_8bit=n_slots_8bit, device=device)
        self.wqkv = self._randn((heads + 2 * kv_heads) * head_dim, hidden) / hidden ** 0.5
        for s in range(chunks):
            self.pc.percache_kv_put(0, s, self._randn(kv_heads, capacity, head_dim), self._randn(kv_heads, capacity, head_dim))
        # one running sum per token that a slot can hold
        self.weights = torch.zeros((chunks + batch, kv_heads, capacity), device=device)
        self.held = np.zeros(batch, np.int32)                              # tokens in each query's own slot
        self.position = np.full(batch, chunks * capacity, np.int32)        # and how many it has seen: cut tokens keep theirs
        self.ids = np.array([[*range(chunks), chunks + b] for b in range(batch)], np.int32)
        self.capacity = capacity

    def _randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.gen.device).to(torch.bfloat16)

    def draft(self):
        """Parents of a tree per query: node 0 is the token accepted last, every other one hangs from one of the few before it."""
        return np.array([[-1] + [int(self.rng.integers(max(0, i - 4), i)) for i in range(1, self.nodes)] for _ in range(self.batch)], np.int32)

    def accept(self, parents):
        """A path from each root to a random node."""
        paths = []
        for row in parents:
            node, path = int(self.rng.integers(0, self.nodes)), []
            while node >= 0:
                path.append(node)
                node = int(row[node])
            paths.append(path[::-1])
        n = np.array([len(p) for p in paths], np.int32)
        return np.array([p + [0] * (int(n.max()) - len(p)) for p in paths], np.int32), n

    def step(self, parents=None):
        pc = self.pc
        parents = self.draft() if parents is None else parents
        used = np.concatenate([np.full((self.batch, self.chunks), self.capacity, np.int32), self.held[:, None]], 1)
        lists = dict(slot_ids=self.ids, used_len=used, n_chunks=(self.chunks + (self.held > 0)).astype(np.int32))   # (an empty slot is not named)
        x = self._randn(self.batch, self.nodes, pc.cfg.hidden)
        q, k, v = pc.percache_qkv_rope_draft(x, self.wqkv, self.position, parents)
        out, lse = pc.percache_attention_draft(0, q, k, v, parents=parents, lse_out=True, **lists)
        path, n_path = self.accept(parents)
        paid = pc.percache_attention_weights(0, q, k, lse, self.weights, self.weights, parents=parents, path=path, n_path=n_path, **lists)
        own = self.chunks + np.arange(self.batch, dtype=np.int32)
        pc.percache_kv_append_path(0, k, v, own, path, n_path=n_path, weights=self.weights, draft_weights=paid)
        self.held += n_path
        self.position += n_path
        full = np.flatnonzero(self.held + self.nodes > self.capacity)      # no room for the longest path of the next step
        if full.size:
            pc.percache_kv_keep(0, own[full], self.budget, self.weights, n_first=self.first, n_last=self.last)
            self.held[full] = np.minimum(self.held[full], self.budget)
        return dict(parents=parents, x=x, q=q, k=k, v=v, out=out, lse=lse, path=path, n_path=n_path, cut=full)

    def close(self):
        self.pc.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--nodes", type=int, default=16)
    a = ap.parse_args()
    d = DraftDecoder(batch=a.batch, nodes=a.nodes)
    for _ in range(10):
        d.step()
    torch.cuda.synchronize()
    t, tokens, cuts = time.perf_counter(), 0, 0
    for _ in range(a.steps):
        r = d.step()
        tokens += int(r["n_path"].sum())
        cuts += len(r["cut"])
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) / a.steps * 1e3
    print(f"{a.batch} queries x {a.nodes} nodes over {d.chunks * d.capacity} shared and up to {d.capacity} own tokens: {ms:.3f} ms a step of one layer, "
          f"{tokens / a.steps / a.batch:.2f} accepted tokens a query and step, {cuts} cuts; held {d.held.tolist()} of {(d.position - d.chunks * d.capacity).tolist()}")
    d.close()


if __name__ == "__main__":
    main()
