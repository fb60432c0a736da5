"""Builds the CUDA library in-tree (sm_100a only) with nvcc; no JIT cache is involved."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libtabed_b200.so")
SOURCES = ["tabed.cu", "pages.cu"]
HEADERS = ["ptx.cuh", "exact_math.cuh", "forward_kernels.cuh", "decide_kernels.cuh", "round_kernel.cuh", "proj_plan.h", "gemm_tc.cuh", "proj_tc.cuh", "attn_tc.cuh", "prompt_attn.cuh", "request_kernels.cuh", "pages.h", "pages_kernels.cuh", "pages_attn.cuh", "pages_attn_tc.cuh", os.path.join("..", "..", "include", "tabed.h")]


def _stale() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, s) for s in SOURCES + HEADERS]
    return any(os.path.getmtime(d) > t for d in deps if os.path.exists(d))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile csrc/*.cu into libtabed_b200.so next to this file; returns its path."""
    if not force and not _stale():
        return LIB_PATH
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    arch = ["-gencode", "arch=compute_100a,code=sm_100a"]
    flags = ["-Xcompiler", "-fPIC", "-O3", "-std=c++17", "-lineinfo"] + arch
    if verbose:
        flags += ["-Xptxas", "-v"]
    # Another process may build at the same time: files of this build's own, and the library appears whole.
    with tempfile.TemporaryDirectory(dir=PKG_DIR, prefix="build") as tmp:
        objects = [os.path.join(tmp, os.path.splitext(s)[0] + ".o") for s in SOURCES]
        linked = os.path.join(tmp, os.path.basename(LIB_PATH))
        runs = [subprocess.Popen([nvcc, "-c"] + flags + ["-o", o, os.path.join(CSRC, s)], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                for s, o in zip(SOURCES, objects)]
        said = [r.communicate()[0] for r in runs]
        if all(r.returncode == 0 for r in runs):
            link = subprocess.run([nvcc, "-shared"] + arch + ["-o", linked] + objects, capture_output=True, text=True)
            runs, said = runs + [link], said + [link.stdout + link.stderr]
        if any(r.returncode != 0 for r in runs):
            raise RuntimeError("nvcc failed:\n" + "".join(said))
        os.replace(linked, LIB_PATH)
    if verbose:
        sys.stderr.write("".join(said))
    return LIB_PATH


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
