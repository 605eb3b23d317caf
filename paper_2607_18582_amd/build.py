"""Build libmure.so (the C-ABI library) and libmure_peaks.so (the measured
copy and MFMA ceilings, ``include/mure_peaks.h``) for gfx950 with hipcc, and
_seq_args.so (the binding's marshalling of torch tensors for
``include/mure_seq.h`` and ``include/mure_attn.h``, host code) with g++, in-tree.

    python -m paper_2607_18582_amd.build        # or build() from Python

Every HIP source is compiled with packed-FP32 instructions disabled; the
objects of ``csrc/`` are linked into ``paper_2607_18582_amd/libmure.so`` and
those of ``peaks/`` into ``paper_2607_18582_amd/libmure_peaks.so``.  The
marshalling module is the only one that uses torch's headers.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libmure.so")
PEAKS = os.path.join(HERE, "peaks")
PEAKS_LIB = os.path.join(HERE, "libmure_peaks.so")
PYEXT_SRC = [os.path.join(HERE, "pyext", f) for f in ("seq_args.cpp", "attn_args.cpp")]
PYEXT_LIB = os.path.join(HERE, "_seq_args.so")
ARCH = "gfx950"

COMMON = ["-O3", "-fPIC", "-std=c++17", f"--offload-arch={ARCH}",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
          "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def sources(d: str = CSRC):
    """The compiled sources of d and its subfolders; their names differ."""
    return sorted(os.path.join(at, f) for at, _, files in os.walk(d) for f in files
                  if f.endswith((".hip", ".cpp")))


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    lang = ["-x", "hip"] if src.endswith(".cpp") else []
    cmd = [hipcc()] + COMMON + lang + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    warn = "\n".join(l for l in r.stderr.splitlines()
                     if "packed-fp32-ops" not in l and l.strip())
    if "warning" in warn:
        sys.stderr.write(warn + "\n")
    return obj


def _link(objs, lib: str, verbose: bool) -> None:
    tmp = lib + ".tmp"
    cmd = [hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, lib)
    if verbose:
        print(f"built {lib}")


def _pyext(verbose: bool) -> None:
    """The torch marshalling module; torch's libraries are those that Python has
    loaded by then."""
    torch = importlib.util.find_spec("torch").submodule_search_locations[0]
    inc = os.path.join(torch, "include")
    tmp = PYEXT_LIB + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall", "-isystem", inc, "-isystem",
           os.path.join(inc, "torch", "csrc", "api", "include"), "-isystem", sysconfig.get_paths()["include"], *PYEXT_SRC,
           "-o", tmp, "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch_hip", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    os.replace(tmp, PYEXT_LIB)
    if verbose:
        print(f"built {PYEXT_LIB}")


def build(verbose: bool = True) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs, psrcs = sources(), sources(PEAKS)
    with ThreadPoolExecutor(max_workers=min(8, len(srcs) + len(psrcs))) as ex:
        ext = ex.submit(_pyext, verbose)
        objs = list(ex.map(_compile, srcs + psrcs))
        ext.result()
    _link(objs[:len(srcs)], LIB, verbose)
    _link(objs[len(srcs):], PEAKS_LIB, verbose)
    return LIB


if __name__ == "__main__":
    build()
