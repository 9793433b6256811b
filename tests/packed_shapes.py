"""Packed calls whose blocks are tall: shapes shared by the GPU tests of the attention and by the CPU test that says which kind of work each of them plans.

A shape is (heads, kv heads, head size, rows of every request, used lengths of every request's chunks or None, capacity).  A request's rows are cut into blocks
of 256 stacked rows (row = token * heads a kv head + head), the last one shorter, of at most 32 where that is what is left; where the 256s fill less than half of the
CUs of a kv head, into 128s or 32s instead.  So the 256s stay where there are few kv heads' CUs for many rows."""
import numpy as np

# many kv heads: short requests fill their CUs
TALL = {
    "32over32x64": (32, 32, 64, [300, 1, 257, 513, 40], [[100, 64, 3], [1, 0, 64], [128, 128, 65], [63, 0, 0], [127, 1, 2]], 128),
    "32over32x128": (32, 32, 128, [290, 2, 260, 511], [[70, 64], [128, 5], [127, 0], [3, 65]], 128),
    "32over8x128": (32, 8, 128, [300, 700, 411], [[190, 64], [65, 1], [192, 130]], 192),
    "14over2x64": (14, 2, 64, [900, 1, 700, 810], [[200, 64], [0, 256], [255, 1], [65, 130]], 256),
    "24over8x128_nothing_cached": (24, 8, 128, [513, 350, 640, 31], None, 64),
    "16over16x64_many_chunks": (16, 16, 64, [600, 1000, 513], [[7] * 70, [64, 1] * 35, [40] * 70], 64),
    "32over8x128_many_chunks": (32, 8, 128, [500, 450, 200], [[64, 5] * 33, [1] * 66, [50, 64] * 33], 64),
}
# few requests: blocks of 128 rows
MIDDLE = {
    "6over2x128": (6, 2, 128, [600], [[511, 300]], 512),
    "8over1x64": (8, 1, 64, [700, 430], [[500, 511, 130], [512, 3, 60]], 512),
    "8over2x128": (8, 2, 128, [513, 300], [[512, 400], [63, 512]], 512),
}


def slots_of(shape):
    """Tokens of every slot, the slots of every request's chunks (or None) and how many of their tokens count."""
    _, _, _, T, used, C = shape
    n_c = len(used[0]) if used else 0
    tokens = [C if s % 3 else max(1, C - 7) for s in range(max(2, len(T) * n_c))]
    if not n_c:
        return tokens, None, None
    ids = np.random.default_rng(len(tokens)).permutation(len(T) * n_c).reshape(len(T), n_c)
    return tokens, ids, np.minimum(np.array(used, np.int32), np.array(tokens, np.int32)[ids])
# calls of the GPU tests: (shape, formats of the chunks, partitions asked for)
CALLS = [(name, f, n) for shapes, splits in ((TALL, (0, 1, 2, 3)), (MIDDLE, (0, 3, 7))) for name in shapes
         for f in (("bf16", "8bit", "mixed") if shapes[name][4] else ("bf16",)) for n in splits]
# requests whose later rows, or whose slots behind the used length, hold what is not finite
RUBBISH = {
    "32over8x128": (32, 8, 128, [300, 130, 600, 64], [[60], [1], [64], [33]], 64),
    "32over32x64": (32, 32, 64, [300, 1, 257, 513], [[100], [64], [127], [1]], 128),
    "14over2x64": (14, 2, 64, [1000, 700, 900], [[63], [0], [64]], 64),
    "16over16x128": (16, 16, 128, [520, 300, 700, 265], [[17], [128], [66], [9]], 128),
}
RUBBISH_CALLS = [(name, f, n) for name in RUBBISH for f in ("bf16", "8bit", "mixed") for n in (0, 1, 3)]
# rows of a projection: heads, kv heads, head size, rows, heads a group of lanes.  On both sides of where the groups take four heads (rows * heads * D / 16 = 1024 a CU) and
# where they take two, past the caches (rows * heads * D * 4 bytes = 160 MiB); head counts that neither divides
ROWS = [
    (14, 2, 128, 1820, 1), (14, 2, 128, 1821, 4), (14, 2, 128, 18204, 4), (14, 2, 128, 18205, 2),
    (3, 3, 128, 3640, 1), (3, 3, 128, 3641, 4), (3, 3, 128, 36408, 4), (3, 3, 128, 36409, 2),
    (14, 2, 64, 3640, 1), (14, 2, 64, 3641, 4), (14, 2, 64, 36408, 4), (14, 2, 64, 36409, 2),
    (6, 2, 64, 6553, 1), (6, 2, 64, 6554, 4), (6, 2, 64, 65536, 4), (6, 2, 64, 65537, 2),
]
