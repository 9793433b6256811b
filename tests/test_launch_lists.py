"""What calls on drafted tokens hand to their kernels, on the CPU: the library's host code, address and undefined-behaviour sanitizers on, over a stand-in
for the HIP runtime (tests/sanitize/launch_driver.cpp) that launches nothing and checks the lists that travel as launch arguments."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_sanitizers import ENV, ROOT, SAN, _clean, _run


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_lists_of_launches_on_a_stand_in_runtime(tmp_path):
    from paper_2601_11553_amd.build import CSRC, FLAGS, HIPCC, SOURCES
    flags = [f for f in FLAGS if f != "-O3"] + [*SAN, "-fno-gpu-sanitize", "--cuda-host-only", "-Wno-division-by-zero"]

    def compile_one(src):
        obj = str(tmp_path / (os.path.splitext(os.path.basename(src))[0] + ".o"))
        _run([HIPCC, *flags, "-x", "hip", "-c", src, "-o", obj])
        return obj

    sources = [os.path.join(CSRC, s) for s in SOURCES] + [os.path.join(ROOT, "tests", "sanitize", "launch_driver.cpp")]
    with ThreadPoolExecutor(max_workers=4) as ex:
        objs = list(ex.map(compile_one, sources))
    # (no device code: its place in the registration stays empty)
    names = subprocess.run(["nm", "-u", *objs], capture_output=True, text=True, check=True).stdout
    empty = [f"-Wl,--defsym={n}=0" for n in sorted(set(re.findall(r"__hip_fatbin_\w+", names)))]
    exe = str(tmp_path / "launch_driver")
    clang = os.path.join(os.path.dirname(os.path.realpath(HIPCC)), "..", "lib", "llvm", "bin", "clang++")
    _run([clang, "-no-pie", *SAN, *objs, *empty, "-o", exe])
    r = subprocess.run([exe], env=ENV, capture_output=True, text=True)
    _clean(r)
    assert r.returncode == 0 and "launch driver: ok" in r.stdout, r.stdout[-3000:]
