"""Refusals of the calls on packed rows and continuations (no effect on anything), other streams, captured calls, long lists and large offsets."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import packed_ref as ref
from paper_2601_11553_amd.binding import Percache, PercacheError

from gpu_util import DEV, bf16, host
from test_gpu_draft import make, stored
from test_gpu_packed import check, packed

pytestmark = pytest.mark.gpu
EINVAL, ESHAPE, ESLOT, ELEN, ENOMEM = -1, -2, -3, -4, -5


def status(call):
    with pytest.raises(PercacheError) as e:
        call()
    return e.value.status


def test_refusals_of_the_packed_attention():
    pc, g, kv = make(51, 4, 2, 64, 64, "bf16", [64, 64, 0])
    q, k, v = packed(g, 4, 2, 64, 30)
    out = torch.full((30, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    call = lambda start, layer=0, **kw: pc.percache_attention_packed(layer, q, k, v, start, attn_out=out, **kw)
    assert status(lambda: call([-1, 5])) == EINVAL
    assert status(lambda: call([0, 5, 4])) == EINVAL
    assert status(lambda: call([0, 31])) == EINVAL
    assert status(lambda: call([0, 30], layer=1)) == ESLOT
    assert status(lambda: call([0, 30], slot_ids=[[3]])) == ESLOT
    assert status(lambda: call([0, 30], slot_ids=[[2]])) == ESLOT
    assert status(lambda: call([0, 30], slot_ids=[[0]], used_len=[[65]])) == ELEN
    assert status(lambda: call([0, 30], slot_ids=[[0]], n_chunks=[2])) == EINVAL
    assert status(lambda: call([0, 30], n_splits=-1)) == EINVAL
    assert status(lambda: call([0, 30], n_splits=65)) == EINVAL
    for bad in (dict(attn_out=out[:29]), dict(lse_out=torch.zeros((4, 29), device=DEV)), dict(slot_ids=[0, 1, 1])):
        with pytest.raises(ValueError):
            pc.percache_attention_packed(0, q, k, v, [0, 15, 30], **bad)
    with pytest.raises(ValueError):
        pc.percache_attention_packed(0, q.transpose(1, 2), k, v, [0, 30])
    with pytest.raises(ValueError):
        pc.percache_attention_packed(0, q, k, v, [0])
    lib, need = pc.lib, pc.lib.percache_packed_workspace_bytes(pc.ctx, 1, 30, 0)
    ws = torch.empty(need + 512, dtype=torch.uint8, device=DEV)
    p = (ws.data_ptr() + 255) // 256 * 256
    start, none = np.array([0, 30], np.int32), np.zeros(1, np.int32)
    at = lambda a: a.ctypes.data
    raw = lambda q_=q.data_ptr(), w=p, n=need, o=out.data_ptr(): lib.percache_attention_packed(pc.ctx, 0, q_, k.data_ptr(), v.data_ptr(), 30, at(start), 1, None, None, at(none), 0, 0, o,
                                                                                              None, w, n, None)
    assert raw(w=None) == ENOMEM and raw(n=need - 1) == ENOMEM and raw(w=p + 128) == EINVAL and raw(q_=q.data_ptr() + 2) == EINVAL and raw(o=None) == EINVAL
    assert lib.percache_attention_packed(None, 0, None, None, None, 0, None, 1, None, None, None, 0, 0, None, None, None, 0, None) == EINVAL
    assert lib.percache_packed_workspace_bytes(pc.ctx, 0, 30, 0) == 0 and lib.percache_packed_max_splits(pc.ctx, 1, -1) == EINVAL
    torch.cuda.synchronize()
    assert (out == 7).all()
    call([3, 3, 3])                   # (nothing to do)
    torch.cuda.synchronize()
    assert (out == 7).all()
    pc.close()


def test_refusals_of_the_rotation():
    pc = Percache(n_layers=1, hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=64, n_slots=1, slot_capacity=64, max_pos=100, device=DEV)
    x, pos = torch.zeros((5, 512), dtype=torch.bfloat16, device=DEV), torch.zeros((2, 5), dtype=torch.int32, device=DEV)
    run = lambda x=x, pos=pos, **kw: pc.percache_qkv_norm_rope(x, pos, **kw)
    assert status(run) == EINVAL                                        # two axes and no list of them
    assert status(lambda: run(axis=np.full(32, 2))) == EINVAL
    assert status(lambda: run(pos=pos[:1].expand(5, 5).contiguous())) == ESHAPE
    assert status(lambda: run(pos=pos[:1], eps=float("nan"))) == EINVAL and status(lambda: run(pos=pos[:1], eps=-1.0)) == EINVAL
    wide = torch.zeros((5, 600), dtype=torch.bfloat16, device=DEV)
    assert status(lambda: run(x=wide[:, 4:516], pos=pos[:1])) == EINVAL      # rows that are not 16-byte aligned
    wide = torch.zeros((5, 517), dtype=torch.bfloat16, device=DEV)
    assert status(lambda: run(x=wide[:, :512], pos=pos[:1])) == EINVAL
    for bad in (dict(x=x.float()), dict(pos=pos[:, :4]), dict(pos=pos[:1].long()), dict(axis=np.zeros(31)), dict(q_norm=x[0]), dict(x=x[:, :500])):
        with pytest.raises(ValueError):
            run(**bad)
    out = pc.percache_qkv_norm_rope(x[:0], pos[:1, :0])
    assert out[0].shape == (4, 0, 64)
    assert pc.lib.percache_qkv_norm_rope(None, None, 0, 0, None, 1, None, None, None, None, 0.0, None, None, None, None) == EINVAL
    pc.close()


def test_refusals_of_the_copies():
    pc, g, kv = make(52, 2, 1, 64, 64, "mixed", [64, 10, 0, 64, 0, 0])
    before = stored(pc)
    fork = pc.percache_kv_fork
    assert status(lambda: fork([0], [6])) == ESLOT and status(lambda: fork([-1], [0])) == ESLOT
    assert status(lambda: fork([2], [0])) == ESLOT                       # an empty source
    assert status(lambda: fork([0], [4])) == ESLOT                       # another format
    assert status(lambda: fork([0, 1], [2, 2])) == EINVAL
    assert status(lambda: fork([1], [2], [11])) == ELEN and status(lambda: fork([1], [2], [0])) == ELEN
    assert status(lambda: fork([0], [2], n_layers=2)) == ESLOT and status(lambda: fork([0], [2], layer0=1, n_layers=1)) == ESLOT
    assert status(lambda: fork([0], [2], n_layers=0)) == ESLOT
    assert status(lambda: fork([0, 1, 2], [1, 2, 0])) == ESLOT
    assert pc.lib.percache_kv_fork(pc.ctx, 0, 1, None, None, None, 1, None) == EINVAL and pc.lib.percache_kv_fork(None, 0, 1, None, None, None, 0, None) == EINVAL
    torch.cuda.synchronize()
    after = stored(pc)
    assert all(np.array_equal(a[x], b[x]) for a, b in zip(before, after) for x in (0, 1))
    pc.close()


def test_refusals_of_the_selection():
    pc = Percache(n_slots=1, slot_capacity=64, max_pos=64, device=DEV)
    x, s = torch.zeros((2, 3, 50), device=DEV), torch.zeros((2, 3), device=DEV)
    run = lambda x=x, s=s, best=4: pc.percache_beam_select(x, s, best)
    assert status(lambda: run(best=0)) == ESHAPE and status(lambda: run(best=65)) == ESHAPE
    assert status(lambda: run(x=torch.zeros((1, 65, 4), device=DEV), s=torch.zeros((1, 65), device=DEV))) == ESHAPE
    assert status(lambda: run(x=torch.zeros((1, 64, 4), device=DEV), s=torch.zeros((1, 64), device=DEV), best=64)) == ESHAPE
    assert status(lambda: run(x=torch.zeros((2, 3, 0), device=DEV))) == ESHAPE
    assert status(lambda: run(x=x[:1, :1].expand(2, 3, 50))) == EINVAL
    for bad in (dict(x=x.half()), dict(x=x.transpose(1, 2)), dict(s=s[:1]), dict(s=s.double()), dict(x=x[0])):
        with pytest.raises(ValueError):
            run(**bad)
    assert [tuple(t.shape) for t in run(x=x[:0], s=s[:0])] == [(0, 4)] * 3
    pc.close()


def test_another_stream_than_the_default_one():
    """Work of a stream stays on it: inputs are made there, behind a long kernel, and the results used there."""
    pc, g, kv = make(53, 4, 2, 128, 128, "mixed", [128] * 4)
    q, k, v = packed(g, 4, 2, 128, 260)
    start, ids = [0, 3, 200, 260], [[0, 3], [1, 2], [2, 0]]
    want = pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids, lse_out=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        slow = torch.randn(4096, 4096, device=DEV)
        for _ in range(20):
            slow = slow @ slow * 1e-2
        q2, k2, v2 = (x + 0 * slow[0, 0].nan_to_num(0.0, 0.0, 0.0).to(torch.bfloat16) for x in (q, k, v))
        got = pc.percache_attention_packed(0, q2, k2, v2, start, slot_ids=ids, lse_out=True)
        logits = torch.matmul(got[0].float(), torch.ones((512, 3000), device=DEV)) + torch.arange(3000, device=DEV) * 1e-2
        best = pc.percache_beam_select(logits[:6].view(2, 3, 3000), torch.zeros((2, 3), device=DEV), 2)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (best[1][:, 0] == 2999).all()
    pc.close()


def test_captured_and_replayed():
    """The four calls in one graph, replayed with other inputs and with eager calls between the replays."""
    pc, g, kv = make(54, 6, 2, 128, 128, "bf16", [128, 100, 128, 60, 128, 128], max_pos=4096)
    n, start, ids = 300, [0, 1, 41, 42, 300], [[0, 1], [1, 2], [2, 3], [3, 0]]
    x = bf16(g.standard_normal((n, 10 * 128)))
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    scores = torch.zeros((2, 2), device=DEV)
    outs = dict(q_out=torch.empty((6, n, 128), dtype=torch.bfloat16, device=DEV), k_out=torch.empty((2, n, 128), dtype=torch.bfloat16, device=DEV),
                v_out=torch.empty((2, n, 128), dtype=torch.bfloat16, device=DEV))

    def run():
        q, k, v = pc.percache_qkv_norm_rope(x, pos, **outs)
        out, lse = pc.percache_attention_packed(0, q, k, v, start, slot_ids=ids, lse_out=True, n_splits=2)
        pc.percache_kv_fork([0, 1], [5, 4])
        return (out, lse, *pc.percache_beam_select(out[:4].view(2, 2, 768), scores, 5))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for i in range(4):
        x.copy_(bf16(g.standard_normal((n, 10 * 128))))
        scores.copy_(torch.rand((2, 2), device=DEV))
        k0, v0 = bf16(g.standard_normal((2, 128, 128))), bf16(g.standard_normal((2, 128, 128)))
        pc.percache_kv_put(0, 0, k0, v0)
        pc.percache_kv_put(0, 5, v0, k0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        assert all(torch.equal(a, b) for a, b in zip(pc.percache_kv_get(0, 5), (k0, v0)))
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    pc.close()


def test_lists_longer_than_a_launchs_arguments():
    """300 requests with chunk lists of their own; and rows so many that the list of blocks alone is long."""
    T = [int(t) for t in np.random.default_rng(55).integers(0, 6, 300)]
    pc, g, kv = make(55, 4, 2, 64, 64, "mixed", [64] * 40, max_pos=1024)
    start = np.concatenate([[0], np.cumsum(T)])
    ids = g.integers(0, 40, (300, 3))
    q, k, v = packed(g, 4, 2, 64, int(start[-1]) + 1)
    for _ in range(3):
        check(pc, kv, q, k, v, start, ids, g.integers(0, 65, (300, 3)))
    T = [5000, 1, 3700]
    start = np.concatenate([[0], np.cumsum(T)])
    q, k, v = packed(g, 4, 2, 64, int(start[-1]))
    out, lse = pc.percache_attention_packed(0, q, k, v, start, lse_out=True)
    one = pc.percache_attention_packed(0, q[:, 5001:].contiguous(), k[:, 5001:].contiguous(), v[:, 5001:].contiguous(), [0, 3700])[0]
    torch.cuda.synchronize()
    # (the same blocks of the same rows, cut into partitions or not: each off by at most 2^-7 of what it adds up, here of max |v|)
    assert (out[5001:].float() - one.float()).abs().max() <= 2.0 ** -6 * v.float().abs().max()
    assert torch.equal(out[5000].view(4, 64), v[:, 5000].repeat_interleave(2, 0)) and torch.isfinite(lse).all()
    pc.close()


def test_a_captured_calls_workspace_stays_when_it_is_outgrown():
    """Warm-up and capture on one stream, then a larger call there: what takes the memory that it gives back is not written by a replay."""
    pc, g, kv = make(57, 4, 2, 64, 64, "bf16", [64] * 4, max_pos=1024)
    q, k, v = packed(g, 4, 2, 64, 600)
    out = torch.zeros((600, 256), dtype=torch.bfloat16, device=DEV)
    small, large = ([0, 300], [0, 600])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    qs, ks, vs = (x[:, :300].contiguous() for x in (q, k, v))

    def call():
        pc.percache_attention_packed(0, qs, ks, vs, small, attn_out=out[:300], n_splits=3)
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    want, size = out.clone(), pc._draft_ws[stream.cuda_stream].numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    with torch.cuda.stream(stream):
        pc.percache_attention_packed(0, q, k, v, large)
        assert pc._draft_ws[stream.cuda_stream].numel() > size
        others = [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for _ in range(3)]
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all((x == 7).all() for x in others)
    pc.close()


def test_a_list_too_long_for_a_captured_call_is_refused():
    """... without harm to the capture: what else is captured runs."""
    pc, g, kv = make(56, 4, 2, 64, 64, "bf16", [64] * 4, max_pos=1024)
    long, short = np.arange(0, 301), [0, 300]
    q, k, v = packed(g, 4, 2, 64, 300)
    out = torch.zeros((300, 256), dtype=torch.bfloat16, device=DEV)
    for start in (long, short):
        pc.percache_attention_packed(0, q, k, v, start, attn_out=out)
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(PercacheError, match="captured"):
            pc.percache_attention_packed(0, q, k, v, long, attn_out=out)
        pc.percache_attention_packed(0, q, k, v, short, attn_out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    pc.close()


def test_offsets_beyond_32_bits():
    """Slots whose elements lie beyond 2^32 bytes of the store, packed rows beyond 2^31 elements of q."""
    pc = Percache(n_layers=1, hidden=64, n_q_heads=2, n_kv_heads=1, head_dim=128, n_slots=3000, slot_capacity=8192, max_pos=16384, device=DEV)   # 6.3 GB each of K and V
    g = torch.Generator(device=DEV).manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)
    for s in (0, 2999):
        pc.percache_kv_put(0, s, r(1, 70, 128), r(1, 70, 128))
    pc.percache_kv_fork([2999, 0], [1499, 2998])
    kv = {s: tuple(host(t).astype(np.float64) for t in pc.percache_kv_get(0, s)) for s in (0, 1499, 2998, 2999)}
    assert all(np.array_equal(kv[a][x], kv[b][x]) for a, b in ((2999, 1499), (0, 2998)) for x in (0, 1))
    q, k, v = r(2, 5, 128), r(1, 5, 128), r(1, 5, 128)
    out, _ = pc.percache_attention_packed(0, q, k, v, [0, 4, 5], slot_ids=[[2999, 1499], [2998, 0]])
    torch.cuda.synchronize()
    h = [host(t).astype(np.float64) for t in (q, k, v)]
    for a, b, s in ((0, 4, (2999, 1499)), (4, 5, (2998, 0))):
        kc, vc = (np.concatenate([kv[i][x] for i in s], 1) for x in (0, 1))
        want, _, size, _ = ref.attend(h[0][:, a:b], h[1][:, a:b], h[2][:, a:b], kc, vc)
        assert (np.abs(host(out[a:b]).astype(np.float64).reshape(b - a, 2, 128) - want) <= (2.0 ** -7 + 2.0 ** -13) * size).all()
    pc.close()
    del pc
    # 9 million packed rows of 2 heads of 128 are 2.3e9 elements of q
    pc = Percache(n_layers=1, hidden=64, n_q_heads=2, n_kv_heads=1, head_dim=128, n_slots=1, slot_capacity=64, max_pos=64, device=DEV)
    n = 9_000_000
    q, k, v = (torch.zeros((h, n, 128), dtype=torch.bfloat16, device=DEV) for h in (2, 1, 1))
    a = n - 40
    q[:, a:], k[:, a:], v[:, a:] = r(2, 40, 128), r(1, 40, 128), r(1, 40, 128)
    out, _ = pc.percache_attention_packed(0, q, k, v, [a, n - 3, n])
    torch.cuda.synchronize()
    h = [host(t[:, a:]).astype(np.float64) for t in (q, k, v)]
    for lo, hi in ((0, 37), (37, 40)):
        none = np.zeros((1, 0, 128))
        want, _, size, _ = ref.attend(h[0][:, lo:hi], h[1][:, lo:hi], h[2][:, lo:hi], none, none)
        got = host(out[a + lo:a + hi]).astype(np.float64).reshape(hi - lo, 2, 128)
        assert (np.abs(got - want) <= (2.0 ** -7 + 2.0 ** -13) * size).all()
    pc.close()
