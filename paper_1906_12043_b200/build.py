"""Build the CUDA libraries in-tree for sm_100a with plain nvcc (cross-compiles without a GPU).

    libcocod.so         the engine (C boundary of include/cocod.h, cocod_mlp.h, cocod_lm.h, cocod_adamw.h)
    libcocod_inputs.so  the device build of the synthetic-input generator (not part of the path)
    _lm_binding.so      Python binding of the language-model operators and of AdamW (host code, g++)
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include"), "-I", CSRC]

TARGETS = {
    "libcocod.so": ["cocod_engine.cu", "cocod_mlp.cu", "cocod_lm.cu", "cocod_lm_rows.cu", "cocod_adamw.cu"],
    "libcocod_inputs.so": ["inputs_gen.cu"],
}


BINDING = "_lm_binding.so"


def _stale(out: str, srcs: list[str], device: bool = True) -> bool:
    if not os.path.exists(out):
        return True
    deps = list(srcs) + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if device and f.endswith((".cuh", ".h"))]
    deps += [os.path.join(ROOT, "include", f) for f in os.listdir(os.path.join(ROOT, "include"))]
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> list[str]:
    nvcc = os.environ.get("NVCC", "nvcc")
    outs = []
    for name, files in TARGETS.items():
        out = os.path.join(HERE, name)
        srcs = [os.path.join(CSRC, f) for f in files]
        if force or _stale(out, srcs):
            tmp = out + f".tmp{os.getpid()}"
            cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + srcs + ["-o", tmp]
            subprocess.check_call(cmd)
            os.replace(tmp, out)
        outs.append(out)
    outs.append(build_binding(force))
    return outs


def build_binding(force: bool = False) -> str:
    out, src = os.path.join(HERE, BINDING), os.path.join(CSRC, "lm_binding.cpp")
    if force or _stale(out, [src], device=False):
        import sysconfig
        import torch
        home = os.path.dirname(torch.__file__)
        cuda = os.path.dirname(os.path.dirname(os.path.realpath(shutil.which(os.environ.get("NVCC", "nvcc")) or "/usr/local/cuda/bin/nvcc")))
        include = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
                   os.path.join(cuda, "include"), sysconfig.get_path("include")]
        tmp = out + f".tmp{os.getpid()}"
        subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", os.path.join(ROOT, "include")] +
                              [a for p in include for a in ("-isystem", p)] + [src, "-o", tmp, "-L", HERE, "-l:libcocod.so",
                              "-L", os.path.join(home, "lib"), "-lc10", "-lc10_cuda", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python",
                              f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-Wl,-rpath,$ORIGIN"])
        os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print("\n".join(build(force="--force" in sys.argv, verbose="-v" in sys.argv)))
