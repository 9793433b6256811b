"""Eviction inside slots around 8192 tokens and above, where the selection reads the weights again in every pass.  Exact, as in test_gpu_keep.py."""
import pytest

from test_gpu_draft import make
from test_gpu_keep import check, weights_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["heavy", "ties", "equal", "odd"])
@pytest.mark.parametrize("in_place", [True, False])
def test_long_slots(in_place, kind):
    lengths = [8191, 8192, 8193, 10048, 9001, 3, 0, 700, 0, 10048]
    pc, g, before = make(26, 2, 1, 64, 10048, "mixed", lengths, max_pos=64)
    w = weights_of(g, kind, (len(lengths), 1, 10048))
    if in_place:
        check(pc, before, w, [0, 1, 2, 3, 4, 9], [8190, 4000, 4001, 10047, 70, 5000], 4, 60)
    else:   # to slots of either format, some of which held something
        check(pc, before, w, [2, 3, 9, 1], [8192, 5003, 10048, 65], 0, 64, dst=[6, 7, 8, 5])
    pc.close()
