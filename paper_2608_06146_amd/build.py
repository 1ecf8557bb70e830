"""Build ``libpadoc_attn.so`` in-tree with hipcc for gfx950, and beside it the
small CPython modules ``_streams`` (where Python's headers are) and ``_rows``
(where PyTorch's are too); without them the package calls the library through
ctypes.

    python -m paper_2608_06146_amd.build            # incremental
    python -m paper_2608_06146_amd.build --force    # rebuild everything

Objects go to ``_build/`` at the repository root; the shared library is
written next to this file, where the Python binding loads it.
"""
from __future__ import annotations

import argparse
import concurrent.futures as cf
import hashlib
import importlib.util
import os
import re
import shutil
import subprocess
import sys
import sysconfig
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libpadoc_attn.so")
STREAMS = os.path.join(PKG, "_streams" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
ARCH = os.environ.get("PADOC_OFFLOAD_ARCH", "gfx950")

STREAMS_SOURCE = "csrc/python/streams.cpp"
ROWS_SOURCE = "csrc/python/rows.cpp"
SOURCES = [
    "csrc/host/plan.cpp",
    "csrc/host/session.cpp",
    "csrc/host/rotary.cpp",
    "csrc/abi.hip",
    "csrc/kernels/tile_mfma_bf16.hip",
    "csrc/kernels/decode_step.hip",
    "csrc/kernels/tile_f32.hip",
    "csrc/kernels/lse_combine.hip",
    "csrc/kernels/bwd.hip",
    "csrc/kernels/append.hip",
    "csrc/kernels/relayout.hip",
    "csrc/kernels/upload.hip",
    "csrc/kernels/rotary.hip",
    "csrc/kernels/copy_blocks.hip",
    "csrc/kernels/cache_e4m3.hip",
    "csrc/kernels/decode_e4m3.hip",
]
# Every header under csrc/ (and the public header) enters each object's
# digest, so an edit to any of them rebuilds every object.
HEADERS = sorted(os.path.relpath(os.path.join(d, f), PKG)
                 for d, _, fs in os.walk(os.path.join(PKG, "csrc")) for f in fs if f.endswith((".hpp", ".h")))

# Packed fp32 VALU forms are kept out of device code on purpose: the
# compiler must not form v_pk_{add,mul,fma}_f32 from scalar fp32 code.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-I", os.path.join(ROOT, "include"),
          "-Wall", "-Wno-unused-function", "-Wno-unused-command-line-argument"]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found (ROCm is required to build libpadoc_attn)")


def _digest(paths) -> str:
    h = hashlib.sha256()
    for p in paths:
        with open(p, "rb") as f:
            h.update(f.read())
    h.update(" ".join(COMMON + DEVICE_FLAGS).encode())
    return h.hexdigest()[:16]


def _compile(cc: str, src: str, force: bool) -> str:
    spath = os.path.join(PKG, src)
    hdrs = [os.path.join(PKG, h) for h in HEADERS] + [os.path.join(ROOT, "include", "padoc_attn.h")]
    tag = _digest([spath] + hdrs)
    obj = os.path.join(BUILD, src.replace("/", "_") + f".{tag}.o")
    if os.path.exists(obj) and not force:
        return obj
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [cc] + COMMON + DEVICE_FLAGS + lang + ["-c", spath, "-o", obj + ".tmp"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(obj + ".tmp", obj)
    return obj


def _compile_streams(cc: str, out: str) -> bool:
    """``_streams`` into file `out`; False where there are no Python headers."""
    inc = sysconfig.get_paths()["include"]
    if not os.path.exists(os.path.join(inc, "Python.h")):
        return False
    cmd = [cc, "-O2", "-std=c++17", "-fPIC", "-Wall", "-shared", "-no-hip-rt", "-I", inc, "-o", out,
           os.path.join(PKG, STREAMS_SOURCE)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return True


def _compile_rows(cc: str, out: str, force: bool) -> bool:
    """``_rows`` into file `out`; False where there are no Python headers or no
    PyTorch headers and libraries for ROCm, and, with a warning, where this
    PyTorch's do not compile or link (the package works without the module)."""
    inc = sysconfig.get_paths()["include"]
    spec = importlib.util.find_spec("torch")
    torch_dir = spec.submodule_search_locations[0] if spec and spec.submodule_search_locations else ""
    needs = [os.path.join(inc, "Python.h")] + [os.path.join(torch_dir, *p.split("/")) for p in
                                               ("include/torch/csrc/autograd/python_variable.h",
                                                "include/c10/hip/HIPStream.h", "lib/libc10_hip.so")]
    if not all(os.path.exists(p) for p in needs):
        return False
    src = os.path.join(PKG, ROWS_SOURCE)
    paths = [inc, os.path.join(ROOT, "include"), os.path.join(torch_dir, "include"),
             os.path.join(torch_dir, "include", "torch", "csrc", "api", "include")]
    cmd = [cc, "-O2", "-std=c++17", "-fPIC", "-Wall", "-shared", "-no-hip-rt", "-DUSE_ROCM", "-D__HIP_PLATFORM_AMD__"]
    cmd += [x for i in paths for x in ("-isystem", i)]
    libs = ["-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip"]
    with open(os.path.join(torch_dir, "version.py")) as f:
        version = re.search(r"^__version__ *= *['\"]([^'\"]+)", f.read(), re.M)
    cmd.append(f'-DPADOC_TORCH_VERSION="{version.group(1) if version else ""}"')  # the module is for this one
    tag = hashlib.sha256(" ".join(cmd + libs).encode() +
                         _digest([src, os.path.join(ROOT, "include", "padoc_attn.h")]).encode()).hexdigest()[:16]
    kept = os.path.join(BUILD, f"rows.{tag}.so")
    if force or not os.path.exists(kept):
        r = subprocess.run(cmd + ["-o", kept + ".tmp", src] + libs, capture_output=True, text=True)
        if r.returncode != 0:
            warnings.warn(f"the module _rows is left out, its compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
            return False
        os.replace(kept + ".tmp", kept)
    shutil.copyfile(kept, out)
    return True


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every source and link the shared library; returns its path.
    What was built before is replaced only once everything has compiled."""
    cc = hipcc()
    os.makedirs(BUILD, exist_ok=True)
    rows = os.path.join(os.path.dirname(STREAMS), "_rows" + STREAMS[STREAMS.index("_streams") + len("_streams"):])
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as ex:
        rows_built = ex.submit(_compile_rows, cc, rows + ".tmp", force)
        objs = list(ex.map(lambda s: _compile(cc, s, force), SOURCES))
        have_rows = rows_built.result()
    tmp = LIB + ".tmp"
    cmd = [cc, "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    have_streams = _compile_streams(cc, STREAMS + ".tmp")
    os.replace(tmp, LIB)
    for have, path in ((have_streams, STREAMS), (have_rows, rows)):
        if have:
            os.replace(path + ".tmp", path)
        elif os.path.exists(path):
            os.remove(path)  # of other sources
    if verbose:
        print(f"built {LIB}")
    return LIB


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--force", action="store_true")
    a = ap.parse_args(argv)
    build(force=a.force, verbose=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
