"""Builds the HIP library in-tree (gfx950 only)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libfikit.so")
MARSHAL = os.path.join(_HERE, "_serve_marshal.so")       # compiled marshalling of the attention calls for Python

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]

UNITS = ["fikit.hip", os.path.join("service", "serve.hip"), os.path.join("service", "around.hip")]        # translation units


def sources():
    return sorted(os.path.join(d, f) for d, _, files in os.walk(CSRC) for f in files if f.endswith((".hip", ".h")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + [os.path.join(ROOT, "include", "fikit.h")]
    return any(os.path.getmtime(s) > t for s in deps)


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objects, compilers = [], []
    for unit in UNITS:                                   # side by side
        obj = os.path.join(CSRC, f"{unit}.tmp{os.getpid()}.o")
        cmd = [hipcc, *HIPCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", "-o", obj, os.path.join(CSRC, unit)]
        if verbose:
            print(" ".join(cmd), flush=True)
        objects.append(obj)
        compilers.append((cmd, subprocess.Popen(cmd)))
    tmp = LIB + f".tmp{os.getpid()}"
    try:
        failed = [cmd for cmd, p in compilers if p.wait() != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.check_call([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objects])
        os.replace(tmp, LIB)
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    return LIB


def build_marshal(force: bool = False, verbose: bool = False) -> str:
    """Host code only, against torch's headers."""
    source = os.path.join(CSRC, "service", "serve_marshal.cpp")
    if not force and os.path.exists(MARSHAL) and all(
            os.path.getmtime(f) <= os.path.getmtime(MARSHAL) for f in (source, os.path.join(ROOT, "include", "fikit.h"))):
        return MARSHAL
    import sysconfig
    import torch
    at = os.path.dirname(torch.__file__)
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", os.path.join(ROOT, "include"), "-I", os.path.join(at, "include"),
           "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"), "-I", sysconfig.get_paths()["include"],
           "-o", tmp, source, "-L", os.path.join(at, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, MARSHAL)
    return MARSHAL


if __name__ == "__main__":
    print(build_library(force=True, verbose=True), build_marshal(force=True, verbose=True))
