"""The 32-bit arithmetic of the relative position bias's map, compiled for the host (tests/host_order/places.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_places(tmp_path):
    exe = tmp_path / "places"
    cmd = [HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-fwrapv", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-I", os.path.join(ROOT, "paper_2110_09132_amd", "csrc"), "-x", "hip",
           os.path.join(ROOT, "tests", "host_order", "places.cpp"), "-o", str(exe)]
    subprocess.run(cmd, check=True, capture_output=True, cwd=str(tmp_path))
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), r.stdout + r.stderr
