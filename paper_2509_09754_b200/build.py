"""Builds liblava.so (sm_100a) with nvcc and, where torch, Python's headers and g++ are there, the paged cache's calls from
Python, both in-tree.  `python -m paper_2509_09754_b200.build`; the library alone, for use from C, needs neither:
`python paper_2509_09754_b200/build.py`."""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB_DIR = os.path.join(PKG, "lib")
LIB_PATH = os.path.join(LIB_DIR, "liblava.so")
CALLS_PATH = os.path.join(LIB_DIR, "_paged_calls.so")

SOURCES = ["lava_api.cu", "score_generic.cu", "budgets.cu", "select.cu", "compact.cu",
           "host_path.cu", "score_sm100.cu", "score_tmem.cu", "score_variants.cu", "cascade.cu", "loss_eval.cu", "decode.cu", "select_shard.cu", "score_static.cu",
           "pages.cu", "compact_pages.cu", "rotary.cu", "decode_pages.cu"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _stale(out: str, deps) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ into one shared library, and the module of calls where its tools are there; returns
    the library's path."""
    os.makedirs(LIB_DIR, exist_ok=True)
    obj_dir = os.path.join(PKG, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers.append(os.path.join(ROOT, "include", "lava.h"))
    objs = []
    for src in SOURCES:
        path = os.path.join(CSRC, src)
        obj = os.path.join(obj_dir, src.replace(".cu", ".o"))
        objs.append(obj)
        if force or _stale(obj, [path] + headers):
            cmd = [_nvcc()] + NVCC_FLAGS + ["-I", os.path.join(ROOT, "include"), "-I", CSRC,
                                            "-c", path, "-o", obj]
            if verbose:
                cmd.insert(1, "-Xptxas=-v")
                print(" ".join(cmd))
            subprocess.run(cmd, check=True)
    if force or _stale(LIB_PATH, objs):
        cmd = [_nvcc(), "-shared", "-o", LIB_PATH] + objs + ["-gencode",
               "arch=compute_100a,code=sm_100a", "-cudart", "static"]
        subprocess.run(cmd, check=True)
    missing = missing_for_calls()
    if missing:
        print("%s: not there; the library is built, the paged cache's calls from Python are not" % ", ".join(missing),
              file=sys.stderr)
    else:
        build_calls(force, verbose)
    return LIB_PATH


def missing_for_calls() -> list:
    """What build_calls() needs and does not find."""
    there = {"torch": importlib.util.find_spec("torch"), "g++": shutil.which("g++"),
             "Python.h": os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h"))}
    return [name for name, x in there.items() if not x]


def build_calls(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/paged_calls.cpp into the module that paged.py loads; returns its path."""
    import torch
    src, header = os.path.join(CSRC, "paged_calls.cpp"), os.path.join(ROOT, "include", "lava.h")
    home = os.path.dirname(torch.__file__)
    if force or _stale(CALLS_PATH, [src, header, os.path.join(home, "version.py")]):
        cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
        cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
               "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
               '-DLAVA_TORCH_VERSION="%s"' % torch.__version__]
        for inc in (os.path.join(ROOT, "include"), os.path.join(home, "include"),
                    os.path.join(home, "include", "torch", "csrc", "api", "include"),
                    sysconfig.get_paths()["include"], os.path.join(cuda, "include")):
            cmd += ["-I", inc]
        # torch's libraries are in the process already when the module is loaded
        cmd += [src, "-o", CALLS_PATH, "-L", LIB_DIR, "-llava", "-Wl,-rpath,$ORIGIN", "-L", os.path.join(home, "lib"),
                "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
        if verbose:
            print(" ".join(cmd))
        subprocess.run(cmd, check=True)
    return CALLS_PATH


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv))
