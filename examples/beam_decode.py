"""Beam search over prompts of different lengths, one layer: the prompts' rows go through a layer packed one behind the other, each request's K/V are
kept in a slot, the slot is handed to the request's beams, and every step extends all beams of all requests by one token, picks the best continuations
and lets the beams' slots change places.

Embeddings, weights and prompts are random here; some prompts hold pictures, whose patches have positions of three axes (time, height, width).  The
products with the weights are the caller's (torch), everything between them is one call.  Run it on the GPU:
python examples/beam_decode.py [--steps N] [--batch B] [--beams K]
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2601_11553_amd.binding import Percache  # noqa: E402


class BeamDecoder:
    """Slots 0 .. chunks - 1: retrieved chunks, shared by all requests; slot chunks + b * beams + i: what beam i of request b has seen itself."""

    def __init__(self, batch=4, beams=4, chunks=3, capacity=512, longest=200, vocab=5000, hidden=1024, heads=16, kv_heads=8, head_dim=128, seed=0, n_slots_8bit=0,
                 device="cuda:0"):
        self.batch, self.beams, self.chunks, self.capacity, self.vocab, self.heads, self.kv_heads, self.D = batch, beams, chunks, capacity, vocab, heads, kv_heads, head_dim
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device=device).manual_seed(seed)
        self.pc = Percache(n_layers=1, hidden=hidden, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, n_slots=chunks + batch * beams, slot_capacity=capacity,
                           max_pos=max(1 << 13, (chunks + 1) * capacity + 64), n_slots_8bit=n_slots_8bit, device=device)
        self.embed = self._randn(vocab, hidden)
        self.wqkv = self._randn((heads + 2 * kv_heads) * head_dim, hidden) / hidden ** 0.5
        self.wo = self._randn(hidden, heads * head_dim) / (heads * head_dim) ** 0.5
        self.q_norm, self.k_norm = (1 + 0.1 * self._randn(head_dim) for _ in "qk")
        for s in range(chunks):
            self.pc.percache_kv_put(0, s, self._randn(kv_heads, capacity, head_dim), self._randn(kv_heads, capacity, head_dim))
        self.axis = (np.arange(head_dim // 2) % 3).astype(np.uint8)
        self.lengths = self.rng.integers(1, longest + 1, batch)
        self.position = np.zeros(batch, np.int64)     # the next position of every request
        self.slots = chunks + np.arange(batch * beams, dtype=np.int32).reshape(batch, beams)

    def _randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device=self.gen.device).to(torch.bfloat16)

    def prompt_positions(self, b):
        """[3, length]: text, and now and then a picture in the middle of it, behind the chunks."""
        n, at, pos = int(self.lengths[b]), self.chunks * self.capacity, []
        while len(pos) < n:
            if self.rng.random() < 0.5:
                pos += [(at + i, at + i, at + i) for i in range(20)]
                at += 20
            else:
                pos += [(at, at + i // 6, at + i % 6) for i in range(24)]
                at += 6
        self.position[b] = max(max(p) for p in pos[:n]) + 1
        return np.array(pos[:n], np.int32).T

    def layer(self, x, pos, start, ids):
        """One layer over packed rows: their attention output, K and V."""
        q, k, v = self.pc.percache_qkv_norm_rope(torch.matmul(x, self.wqkv.t()), torch.from_numpy(np.ascontiguousarray(pos, np.int32)).to(x.device), axis=self.axis,
                                                 q_norm=self.q_norm, k_norm=self.k_norm)
        out, _ = self.pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids)
        self.last = dict(q=q, k=k, v=v, out=out, start=start, ids=ids)
        return out, k, v

    def logits(self, x, out):
        return torch.matmul(x + torch.matmul(out, self.wo.t()), self.embed.t())

    def prompts(self):
        """All prompts in one call; the last row of each opens its beams."""
        B, K = self.batch, self.beams
        start = np.concatenate([[0], np.cumsum(self.lengths)]).astype(np.int32)
        x = self.embed[torch.from_numpy(self.rng.integers(0, self.vocab, int(start[-1]))).to(self.embed.device)]
        pos = np.concatenate([self.prompt_positions(b) for b in range(B)], 1)
        out, k, v = self.layer(x, pos, start, np.tile(np.arange(self.chunks, dtype=np.int32), (B, 1)))
        # the packed rows are one sequence to the slicer, every request a piece of it
        self.pc.percache_kv_slice(0, k, v, start, self.slots[:, 0])
        last = torch.from_numpy(start[1:].astype(np.int64) - 1).to(x.device)
        self.scores = torch.zeros((B, 1), device=x.device)
        self.tokens = np.zeros((B, K, 0), np.int64)
        self.choose(self.logits(x[last], out[last]).view(B, 1, self.vocab))

    def choose(self, logits):
        parent, token, self.scores = self.pc.percache_beam_select(logits, self.scores, self.beams)
        parent, token = parent.cpu().numpy(), token.cpu().numpy()
        # every beam's slot becomes that of the beam it goes on from, all at once.  Where a request has fewer continuations than beams, the others do not exist: a score of
        # -infinity keeps them from being gone on from, their tokens are -1, and their slots are copies of the first beam's, since a row that is computed needs one.
        exists, parent_or_first = parent >= 0, np.maximum(parent, 0)
        src = np.take_along_axis(self.slots, parent_or_first, 1)
        self.pc.percache_kv_fork(src.ravel(), self.slots.ravel())
        before = np.where(exists[..., None], np.take_along_axis(self.tokens, parent_or_first[..., None], 1), -1)
        self.tokens = np.concatenate([before, token[..., None]], 2)
        self.parent, self.token = parent, token

    def step(self):
        """Every beam of every request by one token."""
        B, K = self.batch, self.beams
        x = self.embed[torch.from_numpy(np.maximum(self.token, 0).ravel().astype(np.int64)).to(self.embed.device)]
        pos = np.repeat(self.position, K)
        self.position += 1
        ids = np.concatenate([np.tile(np.arange(self.chunks, dtype=np.int32), (B * K, 1)), self.slots.reshape(-1, 1)], 1)
        out, k, v = self.layer(x, np.stack([pos] * 3), np.arange(B * K + 1, dtype=np.int32), ids)
        self.pc.percache_kv_append_path(0, k.transpose(0, 1).unsqueeze(2).contiguous(), v.transpose(0, 1).unsqueeze(2).contiguous(), self.slots.ravel(),
                                        np.zeros((B * K, 1), np.int32))
        self.choose(self.logits(x, out).view(B, K, self.vocab))

    def close(self):
        self.pc.close()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--beams", type=int, default=4)
    args = ap.parse_args()
    d = BeamDecoder(batch=args.batch, beams=args.beams)
    d.prompts()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(args.steps):
        d.step()
    torch.cuda.synchronize()
    print(f"{args.batch} prompts of {d.lengths.min()} to {d.lengths.max()} tokens, {args.steps} steps of {args.beams} beams: "
          f"{(time.perf_counter() - t) / args.steps * 1e3:.3f} ms a step")
    d.close()


if __name__ == "__main__":
    main()
