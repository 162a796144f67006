"""In-tree build of libharts.so for gfx950 (hipcc, no JIT cache).

Compiles the host planner and the HIP kernels into
``paper_2608_28158_amd/libharts.so``, and the torch binding of the generation
calls into ``_rollout.so`` beside it; both travel with the source tree, so
nothing is built at import time.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT = os.path.join(HERE, "libharts.so")
BINDING = os.path.join(HERE, "_rollout.so")
SOURCES = ["plan.cpp", "semantic.cpp", "mbplan.cpp", "kda_plan.cpp", "gen_plan.cpp", "la.hip", "logp.hip",
           "conv.hip", "attn.hip", "kda.hip", "gen.hip", "step.hip"]

HIP_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 instructions are generated anywhere in the library
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc() -> str:
    return os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def build(verbose: bool = False) -> str:
    """Compile every source and link libharts.so.  Returns its path."""
    obj_dir = os.path.join(HERE, "_build")
    os.makedirs(obj_dir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(obj_dir, src + ".o")
        lang = ["-x", "hip"] if src.endswith(".hip") else []
        _run([hipcc()] + HIP_FLAGS + ["-I", INCLUDE, "-I", CSRC, "-c"] + lang +
             [os.path.join(CSRC, src), "-o", obj], verbose)
        return obj

    # the sources are independent, and the binding of the library: all at once
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        binding = pool.submit(build_binding, verbose)
        objs = list(pool.map(compile_one, SOURCES))
        binding.result()
    tmp = OUT + ".tmp"
    _run([hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC"] + objs + ["-o", tmp], verbose)
    os.replace(tmp, OUT)
    return OUT


def build_binding(verbose: bool = False) -> str:
    """Compile the torch binding of the generation calls (host code, g++; the
    library's functions reach it by address, so it does not link the library)."""
    import torch
    from torch.utils import cpp_extension
    inc = sum((["-isystem", p] for p in cpp_extension.include_paths() + [sysconfig.get_paths()["include"]]), [])
    lib = cpp_extension.library_paths()[0]
    tmp = BINDING + ".tmp"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared",
          f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE] + inc +
         [os.path.join(CSRC, "rollout_ext.cpp"), "-o", tmp, "-L" + lib, "-lc10", "-ltorch_cpu", "-ltorch_python",
          "-Wl,-rpath," + lib], verbose)
    os.replace(tmp, BINDING)
    return BINDING


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout)
        raise RuntimeError(f"build failed: {' '.join(cmd[:3])} ... ({res.returncode})")
    if verbose and res.stdout.strip():
        print(res.stdout)


if __name__ == "__main__":
    print(build(verbose=True))
