"""The shapes of the query-tower operators' launches, at sizes up to their limits
(no GPU needed: launch_shapes.cpp stands in for the runtime's launch functions)."""
import os
import shutil
import subprocess

import pytest

from paper_2609_16175_amd import build, lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_launches_stay_below_2_32_threads(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    lib()   # says so where it is not built
    exe = tmp_path / "launch_shapes"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "launch_shapes.cpp"),
                    "-o", str(exe), "-rdynamic", "-ldl"], check=True, capture_output=True, timeout=300)
    r = subprocess.run([str(exe), build.LIB], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "0 failures" in r.stdout
