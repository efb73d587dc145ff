"""Whether rows overlap (csrc/common.h), built with sanitizers, against every pair of rows
(tests/native/rows_overlap.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_overlap(tmp_path):
    from paper_2608_11688_amd import build
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "rows_overlap")
    cmd = [cxx, "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "-I", "/opt/rocm/include",
           os.path.join(ROOT, "tests", "native", "rows_overlap.cpp"), os.path.join(build.CSRC, "errors.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), (r.stdout[-2000:], r.stderr[-2000:])
