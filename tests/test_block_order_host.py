"""The norms around a block under every lead of one wave over the others, without a GPU: block.hip is compiled for the
host, its launches replaced, and run lane by lane (tests/host_order/block_sim.cpp, fibers.h).  A call in place (h over x,
y over branch; dx over dh, dbranch over dy) has to give what the call with buffers of its own gives."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2110_09132_amd", "csrc")
CLANG = next((c for c in (shutil.which("amdclang++"), "/opt/rocm/llvm/bin/clang++") if c and os.path.exists(c)), None)


def for_host(text):
    """The launches k<<<a>>>(b) as fibers::launch(k, {a})(b)."""
    text, starts = re.subn(r"([A-Za-z_]\w*(?:<[^<>;(){}]*>)?)\s*<<<", r"fibers::launch(\1, {", text)
    text, ends = re.subn(r">>>\(", "})(", text)
    assert starts == ends > 0 and "<<<" not in text
    return text


@pytest.mark.skipif(CLANG is None, reason="clang not found")
def test_calls_in_place(tmp_path):
    with open(os.path.join(CSRC, "block.hip")) as f:
        (tmp_path / "block_host.inc").write_text(for_host(f.read()))
    exe = tmp_path / "block_sim"
    subprocess.run([CLANG, "-O1", "-std=c++17", "-ffp-contract=off", "-U_FORTIFY_SOURCE", "-w", "-I", os.path.join(HERE, "host_order", "stand_in"),
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", str(tmp_path), "-I", os.path.join(HERE, "host_order"),
                    os.path.join(HERE, "host_order", "block_sim.cpp"), "-o", str(exe)], check=True, cwd=str(tmp_path))
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), r.stdout[-3000:] + r.stderr
