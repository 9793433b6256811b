"""What calls on packed rows plan, on the CPU (tests/sanitize/packed_shapes_driver.cpp: the library's host code, sanitizers on, over a stand-in runtime):
which blocks, partitions and formats the shapes of the GPU tests reach, so that no later rule empties these tests unseen; limits of launches and workspaces."""
import os
import re
import shutil
import subprocess
from collections import Counter, namedtuple
from concurrent.futures import ThreadPoolExecutor

import pytest

from packed_shapes import CALLS, MIDDLE, RUBBISH, RUBBISH_CALLS, ROWS, TALL, slots_of
from test_sanitizers import ENV, ROOT, SAN, _clean, _run

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
Item = namedtuple("Item", "rows kind cached fresh partial entries bf16 eight")
FORMATS = {"bf16": 0, "8bit": 1, "mixed": 2}


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    from paper_2601_11553_amd.build import CSRC, FLAGS, HIPCC, SOURCES
    at = tmp_path_factory.mktemp("shapes")
    flags = [f for f in FLAGS if f != "-O3"] + [*SAN, "-fno-gpu-sanitize", "--cuda-host-only", "-Wno-division-by-zero"]

    def compile_one(src):
        obj = str(at / (os.path.splitext(os.path.basename(src))[0] + ".o"))
        _run([HIPCC, *flags, "-x", "hip", "-c", src, "-o", obj])
        return obj

    sources = [os.path.join(CSRC, s) for s in SOURCES] + [os.path.join(ROOT, "tests", "sanitize", "packed_shapes_driver.cpp")]
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, sources))
    # (no device code: its place in the registration stays empty)
    names = subprocess.run(["nm", "-u", *objs], capture_output=True, text=True, check=True).stdout
    empty = [f"-Wl,--defsym={n}=0" for n in sorted(set(re.findall(r"__hip_fatbin_\w+", names)))]
    exe = str(at / "shapes_driver")
    clang = os.path.join(os.path.dirname(os.path.realpath(HIPCC)), "..", "lib", "llvm", "bin", "clang++")
    _run([clang, "-no-pie", *SAN, *objs, *empty, "-o", exe])

    def run(what, lines=()):
        r = subprocess.run([exe, what], env=ENV, capture_output=True, text=True, input="\n".join(lines))
        _clean(r)
        assert r.returncode == 0 and "shapes driver: ok" in r.stdout, r.stdout[-3000:]
        return r.stdout
    return run


def line(shape, formats, n_splits):
    Hq, Hkv, D, T, _, C = shape
    tokens, ids, used = slots_of(shape)
    n = len(tokens)
    words = [Hq, Hkv, D, n, {"bf16": 0, "8bit": n, "mixed": n // 2}[formats], C, *tokens, n_splits, len(T), 0 if ids is None else ids.shape[1], *T]
    if ids is not None:
        words += [int(x) for pair in zip(ids.ravel(), used.ravel()) for x in pair]
    return " ".join(map(str, words))


def plans(driver, calls):
    """The items of every (shape, formats, n_splits)."""
    out = []
    for text in driver("calls", [line(*c) for c in calls]).splitlines():
        if text.startswith("call"):
            assert text.split()[1] == "0", text
            out.append([])
        elif text[0].isdigit():
            out[-1].append(Item(*map(int, text.split())))
    assert len(out) == len(calls) and all(out)
    return out


def classes(items):
    """How many items of more than 128 rows, of more than 32, of more than 16 and of fewer there are, whole and in partitions."""
    return Counter(("tall" if i.rows > 128 else "middle" if i.kind == 0 else "low" if i.rows > 16 else "few", bool(i.partial)) for i in items)


def test_blocks_where_partitions_are_asked_for(driver):
    """The height of the blocks goes by the time that each promises there too: one partition gives what the library's own choice gives where that is uncut, and
    many keys that are cut into several are not walked by blocks of 32 rows."""
    short = {"8over2x128": (8, 2, 128, [128, 64, 96], None, 64), "6over2x64": (6, 2, 64, [120, 100], [[0], [1]], 64)}
    uncut = [(s, f, n) for s in [*short.values(), *(TALL[x] for x in ("32over32x64", "32over32x128", "32over8x128", "24over8x128_nothing_cached"))]
             for f in ("bf16", "mixed") for n in (0, 1)]
    got = plans(driver, uncut)
    for i in range(0, len(got), 2):
        assert not any(x.partial for x in got[i]) and got[i] == got[i + 1], uncut[i]
    assert all(classes(x)["middle", False] for x in got[:8])
    for c, items in zip(many := [(s, f, n) for s in MIDDLE.values() for f in ("bf16", "8bit", "mixed") for n in (3, 7)], plans(driver, many)):
        assert classes(items)["low", True] == 0 and (classes(items)["middle", True] or classes(items)["tall", True]), c


def test_rows_of_a_projection_that_a_launch_holds(driver):
    driver("rows")


def test_workspaces_grow_with_the_call_and_no_further_than_what_is_cut(driver):
    driver("sizes")


def test_what_the_gpu_tests_of_tall_blocks_plan(driver):
    """Every form of the wide blocks is among them: both head sizes, chunks of either format and of both, whole and in partitions, lists of more than 64 entries."""
    shapes = {**TALL, **MIDDLE}
    seen = set()
    for (name, f, n), items in zip(CALLS, plans(driver, [(shapes[name], f, n) for name, f, n in CALLS])):
        c, cut = classes(items), {0: (False, True), 1: (False,)}.get(n, (True,))
        if name in TALL:
            assert any(c["tall", x] for x in cut), (name, f, n, c)
        else:
            assert c["middle", True] or c["tall", True], (name, f, n, c)
        for i in items:
            if i.kind == 0:
                seen.add((shapes[name][2], i.rows > 128, bool(i.partial), "mixed" if i.bf16 and i.eight else "8bit" if i.eight else "bf16" if i.cached else "fresh", i.cached > 0 and i.fresh > 0))
                if i.entries > 64 and i.rows > 128:
                    seen.add((shapes[name][2], "long", "mixed" if i.eight and i.bf16 else "8bit" if i.eight else "bf16"))
    for D in (64, 128):
        for walk in ("bf16", "8bit", "mixed"):
            assert (D, "long", walk) in seen
            for partial in (False, True):
                assert (D, True, partial, walk, True) in seen, (D, partial, walk)
            assert {x for x in seen if x[:2] == (D, False) and x[3] == walk}, (D, walk)
        assert (D, True, True, "fresh", False) in seen and {x for x in seen if x[:2] == (D, False) and x[2]}
    assert (128, True, False, "fresh", False) in seen


def test_what_the_gpu_tests_with_rubbish_plan(driver):
    """Tall blocks, whole and in partitions, over a last tile that later rows and used lengths end."""
    for (name, f, n), items in zip(RUBBISH_CALLS, plans(driver, [(RUBBISH[name], f, n) for name, f, n in RUBBISH_CALLS])):
        c = classes(items)
        assert c["tall", n > 1] or (n == 0 and c["tall", True]), (name, f, n, c)
        assert any(i.rows > 128 and i.fresh and i.cached for i in items), (name, f, n)


def test_forms_of_the_rotation_that_the_gpu_tests_take(driver):
    words = driver("rotations", [" ".join(map(str, c[:4])) for c in ROWS]).split()
    for (Hq, Hkv, D, rows, each), got in zip(ROWS, words[1::2]):
        workgroups = lambda n: (rows * -(-(Hq + 2 * Hkv) // n) * (D // 16) + 255) // 256
        assert int(got) == workgroups(each) and all(workgroups(n) != workgroups(each) for n in {1, 2, 4} - {each}), (Hq, Hkv, D, rows)
    assert {(c[2], c[4]) for c in ROWS} == {(d, n) for d in (64, 128) for n in (1, 2, 4)}
    assert all(any((c[0] + 2 * c[1]) % n and c[4] == n for c in ROWS) for n in (2, 4))
