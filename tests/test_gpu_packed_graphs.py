"""Graphs that hold calls with workspaces -- attention in partitions, the selection of beams, drafted nodes -- replayed beside each other and beside eager calls."""
import pytest
import torch

from gpu_util import DEV, bf16
from test_gpu_draft import make
from test_gpu_packed import packed

pytestmark = pytest.mark.gpu


def test_graphs_replayed_side_by_side():
    """Two graphs captured one after the other (torch captures both on one stream), replayed on two streams at once while a third one runs the calls eagerly."""
    pc, g, kv = make(61, 6, 2, 128, 256, "mixed", [256] * 6, max_pos=4096)
    start, ids = [0, 70, 71, 140], [[0, 3, 5], [1, 2, 0], [4, 1, 3]]
    sets = []
    for _ in range(3):
        q, k, v = packed(g, 6, 2, 128, 140)
        sets.append((q, k, v, bf16(g.standard_normal((8, 6, 20000))), torch.randn((8, 6), device=DEV)))

    def call(q, k, v, logits, scores):
        a, lse = pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids, n_splits=3, lse_out=True)
        return (a, lse, *pc.percache_beam_select(logits, scores, 7))
    want = [call(*x) for x in sets]
    torch.cuda.synchronize()
    graphs, held = [], []
    for x in sets[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(call(*x))
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(8):
        for h in held:
            for t in h:
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for graph, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    graph.replay()
            with torch.cuda.stream(streams[2]):
                eager = call(*sets[2])
        torch.cuda.synchronize()
        for got, w in zip((*held, eager), want):
            assert all(torch.equal(a, b) for a, b in zip(got, w))
    pc.close()


def test_a_graphs_memory_goes_with_it():
    pc, g, kv = make(62, 4, 2, 64, 64, "bf16", [64] * 4, max_pos=1024)
    q, k, v = packed(g, 4, 2, 64, 600)
    out = torch.zeros((600, 256), dtype=torch.bfloat16, device=DEV)
    call = lambda: pc.percache_attention_packed(0, q, k, v, [0, 600], attn_out=out, n_splits=3)
    call()
    torch.cuda.synchronize()
    size, want = pc._draft_ws[pc._raw_stream()].numel(), out.clone()
    torch.cuda.empty_cache()
    before = torch.cuda.memory_allocated(), torch.cuda.memory_reserved()
    for _ in range(3):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.cuda.memory_allocated() - before[0] <= 2 * 512      # (torch's own: a capture makes the generator's seed and offset, blocks of 512 bytes)
        del graph
        torch.cuda.empty_cache()
        assert torch.cuda.memory_reserved() - before[1] < size
    pc.close()
