"""Build the HIP library libemb.so for gfx950 and, where the machine can, the dense operators' short binding,
_native.so (in-tree, next to this file)."""
from __future__ import annotations

import concurrent.futures
import glob
import importlib.util
import os
import shutil
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB_PATH = os.path.join(PKG, "libemb.so")
NATIVE_PATH = os.path.join(PKG, "_native.so")
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", shutil.which("hipcc") or "/opt/rocm/bin/hipcc")
CXXFLAGS = [
    "-O3", "-std=c++17", f"--offload-arch={ARCH}", "-fPIC", "-Wall", "-Wextra", "-Wno-unused-parameter",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", INCLUDE, "-I", CSRC,
]


# Per-file flags.  coalesce.hip: no atomic optimizer (it turns a one-lane
# atomic into a wave-wide form that waits for the result at once, which would
# keep the sort passes' ticket from overlapping their first loads).
# adamw.hip: no fused multiply-adds (8-bit moments are then the same bits
# wherever the formula is evaluated operation by operation).
FILE_FLAGS = {"coalesce.hip": ["-mllvm", "-amdgpu-atomic-optimizer-strategy=None"],
              "adamw.hip": ["-ffp-contract=off"]}


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _compile(src, verbose):
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [HIPCC, *CXXFLAGS, *FILE_FLAGS.get(os.path.basename(src), []), "-c", src, "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = [l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l]
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n" + "\n".join(msgs))
    if msgs and verbose:
        print("\n".join(msgs))
    return obj


def torch_include():
    return os.path.join(importlib.util.find_spec("torch").submodule_search_locations[0], "include")


# What csrc/native.c asks of the machine beside a C compiler: the interpreter's headers, and a torch whose
# DLPack header declares the table of C functions that read a tensor.
_PROBE = """#include <Python.h>
#include <ATen/dlpack.h>
static DLPackDLTensorFromPyObjectNoSync reader;
int main(void) { return reader == NULL ? sizeof(DLPackExchangeAPI) + kDLFloat8_e5m2 + kDLROCM == 0 : 1; }
"""


def build_native(verbose: bool = False):
    """Compile csrc/native.c (host C against the interpreter's headers and torch's copy of dlpack.h), linked
    with libemb.so.  Returns its path, or None where the machine cannot compile it: the package then does
    without."""
    cc = os.environ.get("CC", "gcc")
    include = ["-I", INCLUDE, "-I", sysconfig.get_paths()["include"], "-I", torch_include()]
    try:
        subprocess.run([cc, "-std=c11", *include, "-fsyntax-only", "-x", "c", "-"], input=_PROBE, text=True, check=True,
                       capture_output=True)
    except (OSError, subprocess.CalledProcessError) as e:
        why = (getattr(e, "stderr", None) or str(e)).strip().splitlines()[0]
        print(f"_native.so is not built; the dense operators' calls go through Python and ctypes ({why})", flush=True)
        if os.path.exists(NATIVE_PATH):
            os.remove(NATIVE_PATH)
        return None
    tmp = NATIVE_PATH + ".tmp"
    cmd = [cc, "-O2", "-std=c11", "-Wall", "-Wextra", "-shared", "-fPIC", *include, os.path.join(CSRC, "native.c"),
           "-L", PKG, "-l:libemb.so", "-Wl,-rpath,$ORIGIN", "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, NATIVE_PATH)
    return NATIVE_PATH


def build(verbose: bool = False) -> str:
    """Compile every source in csrc/ and link libemb.so and _native.so.  Always rebuilds."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), sources()))
    tmp = LIB_PATH + ".tmp"
    cmd = [HIPCC, "-shared", f"--offload-arch={ARCH}", "-Wl,--no-undefined", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB_PATH)
    build_native(verbose)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
