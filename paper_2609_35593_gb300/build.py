"""Builds libress.so (the C-ABI library) in-tree with nvcc for sm_103a, and _tensors.so, the
binding's questions about tensors, with the host compiler.

Translation units are compiled in parallel into _build/ and linked into
paper_2609_35593_gb300/libress.so.  A unit is recompiled when it or any header it may
include is newer than its object file, and _tensors.so for another Python or torch as well.
"""
from __future__ import annotations

import glob
import importlib.util
import os
import platform
import shutil
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJDIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libress.so")
TENSORS = os.path.join(HERE, "_tensors.so")
SOURCES = ["ress_abi.cu", "k_select.cu", "k_attn.cu", "k_dot.cu", "k_yagg.cu", "k_oproj.cu",
           "k_norm.cu", "k_rope.cu", "k_rope_bwd.cu", "k_rope_few.cu",
           "k_qkv.cu", "k_flash.cu", "k_flash_bwd.cu", "k_cache.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-Wall",
         "--expt-relaxed-constexpr", "-I", INCLUDE, "-I", CSRC]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libress.so")
    return exe


def _torch_dir() -> str | None:
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec is not None and spec.origin else None


def _tensors_abi(torch: str) -> str:
    """The Python and the torch that _tensors.so is compiled against and linked to: it holds their layouts."""
    with open(os.path.join(torch, "version.py")) as f:
        return f"{sysconfig.get_config_var('SOABI')}\n{torch}\n{f.read()}"


def _tensors_command(src: str, torch: str) -> list[str]:
    """Compiles the one unit that knows torch's tensors (and Python); libress.so knows neither."""
    inc, lib = os.path.join(torch, "include"), os.path.join(torch, "lib")
    includes = ["-I", INCLUDE, "-I", sysconfig.get_paths()["include"], "-isystem", inc, "-isystem",
                os.path.join(inc, "torch", "csrc", "api", "include")]
    return [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", *includes, src, "-o", TENSORS,
            "-L", lib, "-Wl,-rpath," + lib, "-ltorch_python", "-ltorch_cpu", "-lc10"]


def _headers_mtime() -> float:
    hs = glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return max(os.path.getmtime(h) for h in hs)


def build(force: bool = False, verbose: bool = False, extra_flags: list[str] | None = None) -> str:
    """Compile every CUDA translation unit and link libress.so; returns its path."""
    os.makedirs(OBJDIR, exist_ok=True)
    stamp = os.path.join(OBJDIR, "machine")
    machine = platform.machine()
    if not os.path.exists(stamp) or open(stamp).read().strip() != machine:
        force = True  # objects built on another host architecture
    hdr = _headers_mtime()
    flags = FLAGS + (extra_flags or [])
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJDIR, src.replace(".cu", ".o"))
        if force or not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(s), hdr):
            jobs.append([nvcc(), *ARCH, *flags, "-c", s, "-o", o])
    units = len(jobs)
    stamps = {stamp: machine}
    torch = _torch_dir()
    if torch is None:
        print("torch is not installed: libress.so is built without _tensors.so, which binds torch's tensors to it",
              flush=True)
    else:
        s = os.path.join(CSRC, "tensors.cpp")
        abi, abi_stamp = _tensors_abi(torch), os.path.join(OBJDIR, "tensors_abi")
        if (force or not os.path.exists(TENSORS) or os.path.getmtime(TENSORS) < max(os.path.getmtime(s), hdr)
                or not os.path.exists(abi_stamp) or open(abi_stamp).read() != abi):
            jobs.append(_tensors_command(s, torch))
        stamps[abi_stamp] = abi

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"build failed:\n{' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr, flush=True)

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        list(ex.map(run, jobs))
    objs = [os.path.join(OBJDIR, s.replace(".cu", ".o")) for s in SOURCES]
    if units or not os.path.exists(LIB) or os.path.getmtime(LIB) < max(map(os.path.getmtime, objs)):
        run([nvcc(), *ARCH, "-shared", "-o", LIB, *objs])
    for path, text in stamps.items():
        with open(path, "w") as f:
            f.write(text)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose=True))
