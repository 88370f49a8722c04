"""Builds libsnapkv.so for gfx950 in-tree with hipcc (cross-compiles without a GPU), and the compiled part of the binding."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libsnapkv.so")
STEPS = os.path.join(PKG, "_steps.so")   # argument checks and calls of some entries (csrc/snapkv_steps.cpp): host code against torch's headers
SOURCES = ["snapkv_api.hip", "snapkv_geom.hip", "snapkv_fused.hip", "snapkv_wide.hip", "snapkv_select.hip", "snapkv_topk.hip",
           "snapkv_decode.hip", "snapkv_hitrate.hip", "snapkv_append.hip", "snapkv_prompt.hip", "snapkv_paged.hip", "snapkv_mx.hip",
           "snapkv_shared.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# Packed-fp32 instruction selection is switched off for all device code.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-command-line-argument"]


def steps_command() -> list:
    import torch
    from torch.utils import cpp_extension
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *("-I" + p for p in [*cpp_extension.include_paths(), sysconfig.get_paths()["include"]]),
            os.path.join(CSRC, "snapkv_steps.cpp"), "-o", STEPS, "-L" + lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-L" + PKG, "-lsnapkv",
            "-Wl,-rpath,$ORIGIN"]


def missing_for_steps() -> str:
    """What the compiled part of the binding needs and this machine lacks ("": nothing)."""
    if shutil.which("g++") is None:
        return "g++"
    try:
        from torch.utils import cpp_extension
    except ImportError:
        return "torch"
    if not any(os.path.exists(os.path.join(p, "torch", "extension.h")) for p in cpp_extension.include_paths()):
        return "torch's headers"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python's headers"
    return ""


def build_steps(verbose: bool = False) -> None:
    """The compiled part of the binding; where the machine lacks what it needs, none, and the calls that it makes say so when they are made."""
    if os.path.exists(STEPS):
        os.remove(STEPS)
    missing = missing_for_steps()
    if missing:
        print(f"{STEPS} is not built: {missing} not found; the library is complete without it, the binding lacks the steps over microscaled and shared pages",
              flush=True)
        return
    cmd = steps_command()
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)


def build_library(verbose: bool = False) -> str:
    objs = []
    procs = []
    for src in SOURCES:
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        objs.append(obj)
    for cmd, pr in procs:
        out, _ = pr.communicate()
        text = "\n".join(l for l in out.decode().splitlines()
                         if "packed-fp32-ops" not in l)   # the host pass does not know the feature
        if pr.returncode != 0:
            raise RuntimeError("hipcc failed: " + " ".join(cmd) + "\n" + text)
        if verbose and text.strip():
            print(text, flush=True)
    link = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    subprocess.check_call(link)
    build_steps(verbose)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose="-v" in sys.argv))
