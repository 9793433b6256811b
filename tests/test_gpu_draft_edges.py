"""Calls on drafted tokens at the edges of their lists and numbers, against the float64 reference.  Bounds: those of test_gpu_draft.py."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, bf16, host
from test_gpu_draft import make, stored

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,T,live,skipped", [(64, 2000, 1, 2000), (128, 1000, 1, 834), (64, 300, 40, 300)])
@pytest.mark.parametrize("formats", ["bf16", "8bit"])
def test_a_skipped_query_with_a_longer_path_than_any_other(D, T, live, skipped, formats):
    """The skipped query first, in the middle and last; what the others append is what they append without it."""
    pc, g, kv = make(31, 2, 2, D, 64, formats, [10, 0])
    k, v = bf16(g.standard_normal((4, 2, T, D))), bf16(g.standard_normal((4, 2, T, D)))
    path = g.integers(0, T, (4, skipped))
    want = {}
    for slots in ([0, 1, -1, -1], [-1, 0, -7, 1], [-1, -1, 0, 1], [0, -1, 1, -1]):
        n_path = [live if s >= 0 else skipped for s in slots]
        pc.percache_kv_put(0, 0, *(bf16(x) for x in kv[0]))
        pc.percache_kv_evict(0, 1)
        pc.percache_kv_append_path(0, k, v, slots, path, n_path=n_path)
        got = stored(pc)
        for s in (0, 1):
            b = slots.index(s)
            pc.percache_kv_put(0, 0, *(bf16(x) for x in kv[0]))
            pc.percache_kv_evict(0, 1)
            pc.percache_kv_append_path(0, k[b:b + 1].contiguous(), v[b:b + 1].contiguous(), [s], path[b:b + 1, :live])
            alone = stored(pc)[s]
            assert got[s][0].shape[1] == (10 if s == 0 else 0) + live
            assert all(np.array_equal(got[s][x], alone[x]) for x in (0, 1))
            new = host(k[b][:, path[b, :live]]).astype(np.float64)
            if formats == "bf16":
                assert np.array_equal(got[s][0][:, -live:], new)
    pc.close()


def test_a_skipped_query_behind_a_full_list():
    """207 queries with one node each and a skipped one with 200: the last record of the launch."""
    pc, g, kv = make(32, 2, 1, 64, 64, "bf16", [0] * 207)
    k, v = bf16(g.standard_normal((208, 1, 256, 64))), bf16(g.standard_normal((208, 1, 256, 64)))
    path = g.integers(0, 256, (208, 200))
    pc.percache_kv_append_path(0, k, v, list(range(207)) + [-1], path, n_path=[1] * 207 + [200])
    torch.cuda.synchronize()
    for s in (0, 100, 206):
        got = pc.percache_kv_get(0, s)
        assert torch.equal(got[0][:, 0], k[s, :, path[s, 0]]) and torch.equal(got[1][:, 0], v[s, :, path[s, 0]])
    assert all(pc.percache_kv_len(0, s) == 1 for s in range(207))
    pc.close()
