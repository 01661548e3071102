"""In-tree build of the CUDA library (nvcc -> libprofk.so, sm_100a only) and of the binding of its decoding operators."""
from __future__ import annotations

import os
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libprofk.so")
BINDING_PATH = os.path.join(PKG_DIR, "_decode.so")
BINDING_SOURCE = os.path.join(CSRC, "decode_binding.cpp")
SOURCES = ["profk_api.cu", "decode_api.cu", "prompt_api.cu", "chunk_api.cu", "plan.cpp"]


def _newest_source_mtime() -> float:
    paths = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != os.path.basename(BINDING_SOURCE)] + [os.path.join(ROOT, "include", "profk.h")]
    return max(os.path.getmtime(p) for p in paths)


def nvcc_command(extra: list[str] | None = None) -> list[str]:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    cmd = [nvcc, "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
           "-Xcompiler", "-fPIC", "-shared", "--threads", "0", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-o", LIB_PATH] + [os.path.join(CSRC, s) for s in SOURCES]
    return cmd + (extra or []) + os.environ.get("PROFK_NVCC_FLAGS", "").split()


def binding_for() -> str:
    """What the binding is built against: it loads into this interpreter and this torch only."""
    from importlib.metadata import version

    return f"_decode for torch {version('torch')}, {sys.implementation.cache_tag}"


def binding_command() -> list[str]:
    """g++ -> paper_2608_12573_b200/_decode.so, the CPython binding of the decoding operators over torch's tensors."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths, library_paths

    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           f'-DPROFK_BINDING_FOR="{binding_for()}"',
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_paths()["include"]]
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    cmd += [f"-I{p}" for p in include_paths() + [os.path.join(cuda, "include")]]
    cmd += [BINDING_SOURCE, "-o", BINDING_PATH, f"-L{PKG_DIR}", "-l:" + os.path.basename(LIB_PATH), "-Wl,-rpath,$ORIGIN"]
    cmd += [f"-L{p}" for p in library_paths()] + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch", "-ltorch_python"]
    return cmd


def _binding_current() -> bool:
    deps = [BINDING_SOURCE, os.path.join(ROOT, "include", "profk.h")]
    if not os.path.exists(BINDING_PATH) or os.path.getmtime(BINDING_PATH) < max(os.path.getmtime(d) for d in deps):
        return False
    with open(BINDING_PATH, "rb") as f:
        return binding_for().encode() + b"\0" in f.read()


def _build_binding(force: bool) -> None:
    if not force and _binding_current():
        return
    res = subprocess.run(binding_command(), capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("g++ failed building _decode.so")


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile the library and the binding unless up-to-date ones are already in the tree; returns the library's path."""
    if not force and os.path.exists(LIB_PATH) and os.path.getmtime(LIB_PATH) >= _newest_source_mtime():
        _build_binding(force)
        return LIB_PATH
    cmd = nvcc_command(["-Xptxas", "-v"] if verbose else None)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("nvcc failed building libprofk.so")
    if verbose:
        sys.stderr.write(res.stdout + res.stderr)
    _build_binding(force)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
