"""Compile the CUDA library in-tree for sm_100a with nvcc (no JIT cache, no other arch)."""
from __future__ import annotations

import os
import shutil
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
SOURCES = [os.path.join(CSRC, n) for n in ("ckv_api.cu", "ckv_ops.cu", "ckv_step.cu", "ckv_autoscaler.cc", "ckv_global_sim.cc")]
HEADERS = [os.path.join(CSRC, n) for n in ("ckv_cache8.cuh", "ckv_cache_attn.cuh", "ckv_common.cuh", "ckv_device.cuh", "ckv_host.cuh",
                                          "ckv_logits.cuh", "ckv_pagelist.cuh", "ckv_rope.cuh", "ckv_sparse.cuh", "ckv_tables.cuh",
                                          "ckv_verify.cuh")] + \
          [os.path.join(_ROOT, "include", n) for n in ("chiron_kv.h", "chiron_autoscaler.h")]
LIBRARY = os.path.join(_HERE, "libchiron_kv.so")
MARSHAL_SOURCE = os.path.join(CSRC, "ckv_marshal.cpp")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-O3", "-std=c++17", "-lineinfo",
    "-Xcompiler", "-fPIC", "-shared", "-cudart", "static",
    "-I", os.path.join(_ROOT, "include"), "-I", CSRC,
]


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found; the CUDA library cannot be built")
    return exe


def is_stale() -> bool:
    if not os.path.exists(LIBRARY):
        return True
    built = os.path.getmtime(LIBRARY)
    return any(os.path.getmtime(p) > built for p in SOURCES + HEADERS)


def marshal_path() -> str:
    """Where the extension module lies.  It uses Python's and torch's own structures, so its name holds both versions:
    a module built for others is neither loaded nor taken for up to date."""
    import sysconfig

    import torch
    return os.path.join(_HERE, "_marshal.torch-%s%s" % (torch.__version__, sysconfig.get_config_var("EXT_SUFFIX")))


def build_marshal(force: bool = False) -> str:
    """Build the extension module, the argument marshalling of the hot calls (g++, Python's and torch's headers)."""
    sources = [MARSHAL_SOURCE, os.path.join(_ROOT, "include", "chiron_kv.h")]
    path = marshal_path()
    if force or not os.path.exists(path) or any(os.path.getmtime(p) > os.path.getmtime(path) for p in sources):
        import sysconfig

        import torch
        home = os.path.dirname(torch.__file__)
        tmp = path + ".tmp.%d" % os.getpid()
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
               "-I", os.path.join(_ROOT, "include"), "-I", sysconfig.get_paths()["include"],
               "-isystem", os.path.join(home, "include"), "-isystem", os.path.join(home, "include", "torch", "csrc", "api", "include"),
               "-o", tmp, MARSHAL_SOURCE, "-L", _HERE, "-l:libchiron_kv.so", "-Wl,-rpath,$ORIGIN",
               "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch", "-lc10", "-Wl,-rpath," + os.path.join(home, "lib")]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("g++ failed:\n%s\n%s" % (res.stdout, res.stderr))
        os.replace(tmp, path)
    return path


def build(force: bool = False, verbose: bool = False) -> str:
    """Build libchiron_kv.so (and the extension module) if missing or older than their sources; return its path."""
    if force or is_stale():
        tmp = LIBRARY + ".tmp.%d" % os.getpid()
        cmd = [_nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("nvcc failed:\n%s\n%s" % (res.stdout, res.stderr))
        if verbose:
            print(res.stderr)
        os.replace(tmp, LIBRARY)
    build_marshal(force)
    return LIBRARY


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
