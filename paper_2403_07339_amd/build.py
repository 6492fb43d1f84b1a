"""Builds libimunpack.so (gfx950) in-tree with hipcc, and the module that marshals torch tensors for it (host code) with the C++ compiler."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libimunpack.so")
SOURCES = ["api.hip", "percentile.hip", "quantize.hip", "plan.hip", "unpack.hip", "gemm.hip", "batched.hip", "norm.hip", "adamw.hip", "xent.hip"]
TENSORS = os.path.join(HERE, "_tensors.so")
CXX = os.environ.get("CXX", "g++")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-fast-math",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-result"]


def _tensors_command() -> list[str]:
    """The compiler's call for _tensors.so: a Python extension on torch's headers."""
    import torch
    from torch.utils import cpp_extension
    libs = cpp_extension.library_paths()
    return [CXX, "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *[f"-isystem{p}" for p in cpp_extension.include_paths()], "-isystem" + sysconfig.get_paths()["include"], os.path.join(CSRC, "tensors.cpp"), "-o", TENSORS,
            *[f"-L{p}" for p in libs], *[f"-Wl,-rpath,{p}" for p in libs], "-lc10", "-ltorch_cpu", "-ltorch_python"]


def build(verbose: bool = False) -> str:
    objs = []
    procs = []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for src in SOURCES:
        obj = os.path.join(HERE, "_build", src.replace(".hip", ".o"))
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    procs.append(("tensors.cpp", subprocess.Popen(_tensors_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
    failed = False
    for src, pr in procs:
        out = pr.communicate()[0].decode()
        text = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l and l.strip())
        if pr.returncode != 0:
            failed = True
            print(f"--- {src} failed\n{out}", file=sys.stderr)
        elif verbose and text:
            print(f"--- {src}\n{text}")
    if failed:
        raise RuntimeError("the compiler failed")
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
